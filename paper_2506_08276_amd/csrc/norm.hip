// Dropout, and LayerNorm with its gradient, over matrices of rows (gfx950).
#include <algorithm>

#include "rows.h"
#include "wave.h"

namespace {

// out = residual + dropout(x).  One access of eight elements per thread and step: one generator call makes the eight's numbers, and no row length leaves lanes idle.
// Bound by memory: 131 072 x 768 bf16 with residual 112 us, 5.4 TB/s; a dozen rows take a launch, 7.6 us.
template <class T, bool DROP, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(const T *x, int64_t ldx, const T *res, int64_t ldr, T *out, int64_t ldo, int rows, int cols,
                                                      int streaming, Drop drop)
{
    const int chunks = (cols + 7) >> 3;
    const uint64_t first = (uint64_t)blockIdx.x * 256 + threadIdx.x, step = (uint64_t)gridDim.x * 256;
    int64_t row = (int64_t)(first / chunks);
    int chunk = (int)(first % chunks);
    const int64_t row_step = (int64_t)(step / chunks);
    const int chunk_step = (int)(step % chunks);
    while (row < rows) {
        const int n = min(8, cols - chunk * 8);
        Raw8<T> a, r;
        a.load(x + row * ldx + chunk * 8, n);
        if constexpr (RES) r.load(res + row * ldr + chunk * 8, n);
        f32x8 v = a.wide();
        if constexpr (DROP) v = dropped(v, drop, chunk, row);
        if constexpr (RES) v += r.wide();
        a.round(v);
        a.store(out + row * ldo + chunk * 8, n, streaming);
        row += row_step;
        chunk += chunk_step;
        if (chunk >= chunks) {
            chunk -= chunks;
            ++row;
        }
    }
}

// Sum over the LPR lanes of a row, in all of them: part of a wavefront (of neighbouring lanes), one, or several; for those `slot` is one of two alternating
// places, so that one barrier per sum is enough.
template <int LPR>
__device__ inline float row_sum(float v, float *shared, int slot)
{
    if constexpr (LPR < 64) {
        if constexpr (LPR == 32) {
            const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        }
        v += __uint_as_float(dpp_mov<DPP_ROW_ROR8>(__float_as_uint(v)));
        v += __uint_as_float(dpp_mov<DPP_ROW_ROR4>(__float_as_uint(v)));
        v += __uint_as_float(dpp_mov<DPP_ROW_ROR2>(__float_as_uint(v)));
        v += __uint_as_float(dpp_mov<DPP_QUAD_XOR1>(__float_as_uint(v)));
    } else {
        v = wave_sum(v);
    }
    if constexpr (LPR > 64) {
        constexpr int WPR = LPR / 64;
        float *s = shared + slot * WPR;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) v += s[i];
    }
    return v;
}

// Which rows a thread works on: LPR lanes per row, blocks of 256 threads.
template <int LPR>
struct RowsOf {
    static constexpr int PER_BLOCK = 256 / LPR;
    static __device__ inline int at() { return threadIdx.x % LPR; }  // the thread's first access of a row
    static __device__ inline int64_t first()
    {
        // the same in a whole wavefront or block: a scalar
        if constexpr (LPR == 256) return blockIdx.x;
        else if constexpr (LPR == 64) return (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        else return (int64_t)blockIdx.x * PER_BLOCK + threadIdx.x / LPR;
    }
};

__device__ inline float sum8(const f32x8 &v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

// t = residual + dropout(x); out = (t - mean) rstd gamma + beta.  LPR lanes per row, NC accesses of eight elements per lane.
// Mean first, then the squares of what is left, both from registers in 32 bits: rows whose mean is large lose nothing, and x is read once.  The next row is on its
// way while this one is added up, where there is one: eight blocks per compute unit, so from 8192 rows of a wavefront each on (4099 x 1021 fp32: 9.6 us, 3.5 TB/s).  Bound by
// memory: 131 072 x 768 bf16 with dropout, residual, total and statistics 148 us, 5.4 TB/s; a dozen rows 9.1 us.
template <class T, int LPR, int NC, bool DROP>
__global__ __launch_bounds__(256) void layernorm_kernel(const T *x, int64_t ldx, const T *res, int64_t ldr, int rows, int cols,
                                                        const float *gamma, const float *beta, float eps, T *out, int64_t ldo, T *total,
                                                        int64_t ldt, float *mean_out, float *rstd_out, int streaming, Drop drop)
{
    __shared__ float shared[2 * 2 * 4];
    constexpr int STRIDE = LPR;
    const int at = RowsOf<LPR>::at();
    int64_t row = RowsOf<LPR>::first();
    const int64_t step = (int64_t)gridDim.x * RowsOf<LPR>::PER_BLOCK;
    if (row >= rows) return;  // all lanes of the row

    int n[NC];
    f32x8 g[NC], b[NC];
    Raw8<T> xs[NC], rs[NC];
    auto request = [&](int64_t r) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (n[i] > 0) {
                xs[i].load(x + r * ldx + (at + i * STRIDE) * 8, n[i]);
                if (res) rs[i].load(res + r * ldr + (at + i * STRIDE) * 8, n[i]);
            }
    };
#pragma unroll
    for (int i = 0; i < NC; ++i) n[i] = min(8, cols - (at + i * STRIDE) * 8);
    request(row);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        g[i] = b[i] = f32x8{};
        if (n[i] > 0) {
            Raw8<float> v;
            v.load(gamma + (at + i * STRIDE) * 8, n[i]);
            g[i] = v.v;
            v.load(beta + (at + i * STRIDE) * 8, n[i]);
            b[i] = v.v;
        }
    }
    const float inv = 1.f / (float)cols;
    for (int slot = 0;; slot ^= 2) {
        f32x8 t[NC];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            t[i] = f32x8{};
            if (n[i] > 0) {
                t[i] = xs[i].wide();
                if constexpr (DROP) t[i] = dropped(t[i], drop, at + i * STRIDE, row);
                if (res) t[i] += rs[i].wide();
                s += sum8(t[i]);  // what is beyond the row's end is 0
            }
        }
        const int64_t next = row + step;
        if (next < rows) request(next);
        const float mean = row_sum<LPR>(s, shared, slot) * inv;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (n[i] > 0) {
                if (total) {
                    Raw8<T> v;
                    v.round(t[i]);
                    v.store(total + row * ldt + (at + i * STRIDE) * 8, n[i], streaming);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    t[i][j] -= mean;
                    q += j < n[i] ? t[i][j] * t[i][j] : 0.f;
                }
            }
        const float rstd = rsqrtf(row_sum<LPR>(q, shared, slot + 1) * inv + eps);
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (n[i] > 0) {
                Raw8<T> v;
                v.round(t[i] * rstd * g[i] + b[i]);
                v.store(out + row * ldo + (at + i * STRIDE) * 8, n[i], streaming);
            }
        if (mean_out && at == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
        if (next >= rows) break;
        row = next;
    }
}

// dt = rstd (gy - mean(gy) - xhat mean(gy xhat)) + dtotal with gy = dout gamma, xhat = (t - mean) rstd; dx = dropout's gradient of dt.  Every block adds up
// dout xhat and dout over its rows in registers and writes one row of `partial` [blocks][2][cols]: no atomics, the same order in every call.  Two blocks per compute
// unit: each more adds a row to sum (131 072 x 768 bf16: 162 us, with four 170).  Bound by memory: with dropout, without dtotal 153 to 162 us by card, 5.0 to 5.3 TB/s.
template <class T, int LPR, int NC, bool DROP>
__global__ __launch_bounds__(256) void layernorm_grad_kernel(const T *dout, int64_t ldd, const T *total, int64_t ldt, int rows, int cols,
                                                             const float *gamma, const float *mean_in, const float *rstd_in, const T *dtotal,
                                                             int64_t lde, T *dres, int64_t ldr, T *dx, int64_t ldx, float *partial,
                                                             int streaming, Drop drop)
{
    __shared__ float shared[2 * 2 * 4];
    extern __shared__ float column[];  // more than one row per block: [2][NC * LPR * 8]
    constexpr int STRIDE = LPR;
    const int at = RowsOf<LPR>::at();
    int64_t row = RowsOf<LPR>::first();
    const int64_t step = (int64_t)gridDim.x * RowsOf<LPR>::PER_BLOCK;

    int n[NC];
    f32x8 g[NC], dg[NC], db[NC];
    Raw8<T> ds[NC], ts[NC], es[NC];
    float mean = 0.f, rstd = 0.f;
    auto request = [&](int64_t r) {
        mean = mean_in[r];
        rstd = rstd_in[r];
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (n[i] > 0) {
                ds[i].load(dout + r * ldd + (at + i * STRIDE) * 8, n[i]);
                ts[i].load(total + r * ldt + (at + i * STRIDE) * 8, n[i]);
                if (dtotal) es[i].load(dtotal + r * lde + (at + i * STRIDE) * 8, n[i]);
            }
    };
#pragma unroll
    for (int i = 0; i < NC; ++i) n[i] = min(8, cols - (at + i * STRIDE) * 8);
    if (row < rows) request(row);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        g[i] = dg[i] = db[i] = f32x8{};
        if (n[i] > 0) {
            Raw8<float> v;
            v.load(gamma + (at + i * STRIDE) * 8, n[i]);
            g[i] = v.v;
        }
    }
    const float inv = 1.f / (float)cols;
    for (int slot = 0; row < rows; row += step, slot ^= 2) {
        f32x8 gy[NC], xhat[NC], e[NC];
        float s = 0.f, q = 0.f;
        const float r = rstd;
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (n[i] > 0) {
                const f32x8 d = ds[i].wide();
                xhat[i] = (ts[i].wide() - mean) * r;
#pragma unroll
                for (int j = 0; j < 8; ++j) xhat[i][j] = j < n[i] ? xhat[i][j] : 0.f;
                gy[i] = d * g[i];
                dg[i] += d * xhat[i];
                db[i] += d;
                s += sum8(gy[i]);
                q += sum8(gy[i] * xhat[i]);
                if (dtotal) e[i] = es[i].wide();
            }
        if (row + step < rows) request(row + step);
        s = row_sum<LPR>(s, shared, slot) * inv;
        q = row_sum<LPR>(q, shared, slot + 1) * inv;
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (n[i] > 0) {
                f32x8 dt = (gy[i] - (s + xhat[i] * q)) * r;
                if (dtotal) dt += e[i];
                Raw8<T> v;
                v.round(dt);
                v.store(dres + row * ldr + (at + i * STRIDE) * 8, n[i], streaming);
                if constexpr (DROP) {
                    v.round(dropped(dt, drop, at + i * STRIDE, row));
                    v.store(dx + row * ldx + (at + i * STRIDE) * 8, n[i], streaming);
                }
            }
    }
    float *mine = partial + (size_t)blockIdx.x * 2 * cols;
    if constexpr (LPR <= 64) {  // the sums of the block's rows, in order
        const int mine_of = threadIdx.x / LPR;
        for (int w = 0; w < 256 / LPR; ++w) {
            if (mine_of == w)
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    f32x8 *to = reinterpret_cast<f32x8 *>(column) + (at + i * LPR);
                    to[0] = w ? to[0] + dg[i] : dg[i];
                    to[NC * LPR] = w ? to[NC * LPR] + db[i] : db[i];
                }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += 256) {
            mine[c] = column[c];
            mine[cols + c] = column[NC * LPR * 8 + c];
        }
    } else {
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (n[i] > 0) {
                Raw8<float> v;
                v.v = dg[i];
                v.store(mine + (at + i * STRIDE) * 8, n[i]);
                v.v = db[i];
                v.store(mine + cols + (at + i * STRIDE) * 8, n[i]);
            }
    }
}

// dgamma and dbeta from the blocks' sums: 16 columns per block, four lanes to a row of them, 256 rows at a time.  Always in the same order.  512 sums of 768 columns
// (3 MB, in the caches): 5.1 us, most of it the launch and the sums' way through LDS.
__global__ __launch_bounds__(1024) void column_sum_kernel(const float *partial, int blocks, int cols, float *dgamma, float *dbeta)
{
    __shared__ float sums[256][17];
    const int tx = threadIdx.x & 3, ty = threadIdx.x >> 2, c = blockIdx.x * 16 + tx * 4, width = 2 * cols;
    f32x4 s = {};
    for (int i = ty; i < blocks; i += 256) {
        f32x4 v = {};
        if (c + 4 <= width) {
            __builtin_memcpy(&v, partial + (size_t)i * width + c, sizeof(v));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = c + e < width ? partial[(size_t)i * width + c + e] : 0.f;
        }
        s += v;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[ty][tx * 4 + e] = s[e];
    for (int half = 128; half >= 1; half >>= 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < half * 16; i += 1024) sums[i >> 4][i & 15] += sums[(i >> 4) + half][i & 15];
    }
    __syncthreads();
    if (threadIdx.x < 16) {
        const int to = blockIdx.x * 16 + threadIdx.x;
        if (to < cols) dgamma[to] = sums[0][threadIdx.x];
        else if (to < width) dbeta[to - cols] = sums[0][threadIdx.x];
    }
}

constexpr int MAX_COLS = 4 * 64 * 8 * 4;  // of a LayerNorm's row

// A row's lanes and accesses per lane: 16 lanes up to 128 columns, 32 up to 256, a wavefront up to 2048, a block beyond.  131 072 rows in bf16 with dropout, this and a
// wavefront per row: 128 columns 18.5 and 47 us (gradient 30 and 82), 256 columns 35 and 47 (59 and 85); over 4096 rows and fewer both take a launch's time.
template <class F>
int with_row_shape(int cols, F f)
{
    const int chunks = (cols + 7) / 8;
    if (chunks <= 16) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (chunks <= 32) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    if (chunks <= 64) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    if (chunks <= 128) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if (chunks <= 192) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 3>());
    if (chunks <= 256) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
    if (chunks <= 512) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
}

template <class F>
int with_type(int dtype, F f)
{
    if (dtype == LEANN_F32) return f((float *)nullptr);
    if (dtype == LEANN_BF16) return f((bf16_t *)nullptr);
    return f((f16_t *)nullptr);
}

// Outputs that the caches would not hold until they are read go past them: dropout + LayerNorm, dropout and the gradient in a row over 131 072 x 768 bf16 take 421
// instead of 436 us, over 65 536 rows 215 and 217; over 16 384 rows it would be 64 instead of 62.
int streams(int64_t rows, int64_t cols, size_t size) { return (double)rows * cols * size >= 96e6; }

int check_matrix(const char *call, int64_t rows, int64_t cols, int dtype)
{
    if (rows < 0 || cols < 1 || (dtype != LEANN_F32 && dtype != LEANN_BF16 && dtype != LEANN_F16)) {
        leann_set_error("%s: negative row count, no columns or unknown type", call);
        return LEANN_EINVAL;
    }
    if (rows > 0x7fffffffll || cols > 0x7fffffffll - 8) {
        leann_set_error("%s: %lld x %lld elements are not covered (rows and columns below 2^31)", call, (long long)rows, (long long)cols);
        return LEANN_ESHAPE;
    }
    return LEANN_OK;
}

int check_rows(const char *call, const char *what, const void *p, int64_t ld, int64_t cols)
{
    if (!p) {
        leann_set_error("%s: %s is null", call, what);
        return LEANN_EINVAL;
    }
    if (ld < cols) {
        leann_set_error("%s: rows of %s are %lld elements apart and %lld long", call, what, (long long)ld, (long long)cols);
        return LEANN_ESHAPE;
    }
    return LEANN_OK;
}

int make_drop(const char *call, const leann_dropout_desc *d, Drop *out)
{
    *out = Drop{0, 0, 0, 0, 0, 1.f};
    if (!d) return LEANN_OK;
    if (!(d->p >= 0.f && d->p <= 1.f)) {
        leann_set_error("%s: dropout rate outside [0, 1]", call);
        return LEANN_EINVAL;
    }
    const uint32_t below = (uint32_t)lrintf(d->p * 65536.f);
    *out = Drop{(uint32_t)d->seed, (uint32_t)(d->seed >> 32), (uint32_t)d->offset, (uint32_t)(d->offset >> 32), below,
                below < 65536 ? 65536.f / (float)(65536 - below) : 0.f};
    return LEANN_OK;
}

int launched(const char *call)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return LEANN_OK;
    leann_set_error("%s: launch failed: %s", call, hipGetErrorString(e));
    return LEANN_EDEVICE;
}

}  // namespace

extern "C" {

int leann_dropout(leann_ctx *ctx, const void *x_dev, int64_t ldx, const void *residual_dev, int64_t ldr, int64_t rows, int64_t cols, int dtype,
                  const leann_dropout_desc *drop, void *out_dev, int64_t ldo)
{
    static const char *call = "leann_dropout";
    if (!ctx || !drop) {
        leann_set_error("%s: null context or dropout", call);
        return LEANN_EINVAL;
    }
    LEANN_TRY(check_matrix(call, rows, cols, dtype));
    Drop d;
    LEANN_TRY(make_drop(call, drop, &d));
    if (rows == 0) return LEANN_OK;
    LEANN_TRY(check_rows(call, "x", x_dev, ldx, cols));
    LEANN_TRY(check_rows(call, "out", out_dev, ldo, cols));
    if (residual_dev) LEANN_TRY(check_rows(call, "residual", residual_dev, ldr, cols));
    LEANN_HIP(hipSetDevice(ctx->device));
    const int64_t items = rows * ((cols + 7) / 8);
    const unsigned grid = (unsigned)std::min<int64_t>((items + 255) / 256, (int64_t)ctx->num_cus * 16);
    return with_type(dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, ctx->stream, (const T *)x_dev, ldx, (const T *)residual_dev, ldr, (T *)out_dev, ldo,
                               (int)rows, (int)cols, streams(rows, cols, sizeof(T)), d);
        };
        if (d.below) residual_dev ? go(dropout_kernel<T, true, true>) : go(dropout_kernel<T, true, false>);
        else residual_dev ? go(dropout_kernel<T, false, true>) : go(dropout_kernel<T, false, false>);
        return launched(call);
    });
}

int leann_layernorm(leann_ctx *ctx, const void *x_dev, int64_t ldx, const void *residual_dev, int64_t ldr, int64_t rows, int32_t cols, int dtype,
                    const leann_dropout_desc *drop, const float *gamma_dev, const float *beta_dev, float eps, void *out_dev, int64_t ldo,
                    void *total_dev, int64_t ldt, float *mean_dev, float *rstd_dev)
{
    static const char *call = "leann_layernorm";
    if (!ctx || !gamma_dev || !beta_dev || !mean_dev != !rstd_dev) {
        leann_set_error("%s: null context, scale or shift, or only one of mean and rstd", call);
        return LEANN_EINVAL;
    }
    LEANN_TRY(check_matrix(call, rows, cols, dtype));
    if (!(eps > 0.f) || !(eps < INFINITY)) {
        leann_set_error("%s: eps has to be positive and finite", call);
        return LEANN_EINVAL;
    }
    if (cols > MAX_COLS) {
        leann_set_error("%s: rows of %d elements are not covered (at most %d)", call, cols, MAX_COLS);
        return LEANN_ESHAPE;
    }
    Drop d;
    LEANN_TRY(make_drop(call, drop, &d));
    if (rows == 0) return LEANN_OK;
    LEANN_TRY(check_rows(call, "x", x_dev, ldx, cols));
    LEANN_TRY(check_rows(call, "out", out_dev, ldo, cols));
    if (residual_dev) LEANN_TRY(check_rows(call, "residual", residual_dev, ldr, cols));
    if (total_dev) LEANN_TRY(check_rows(call, "total", total_dev, ldt, cols));
    LEANN_HIP(hipSetDevice(ctx->device));
    return with_type(dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        return with_row_shape(cols, [&](auto lpr, auto nc) {
            constexpr int LPR = decltype(lpr)::value, NC = decltype(nc)::value;
            const int64_t blocks = (rows + 256 / LPR - 1) / (256 / LPR);
            const unsigned grid = (unsigned)std::min<int64_t>(blocks, (int64_t)ctx->num_cus * 8);
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, ctx->stream, (const T *)x_dev, ldx,
                                   (const T *)residual_dev, ldr, (int)rows, (int)cols, gamma_dev, beta_dev, eps, (T *)out_dev, ldo, (T *)total_dev,
                                   ldt, mean_dev, rstd_dev, streams(rows, cols, sizeof(T)), d);
            };
            if (d.below) go(layernorm_kernel<T, LPR, NC, true>);
            else go(layernorm_kernel<T, LPR, NC, false>);
            return launched(call);
        });
    });
}

int leann_layernorm_backward(leann_ctx *ctx, const void *dout_dev, int64_t ldd, const void *total_dev, int64_t ldt, int64_t rows, int32_t cols,
                             int dtype, const float *gamma_dev, const float *mean_dev, const float *rstd_dev, const void *dtotal_dev, int64_t lde,
                             const leann_dropout_desc *drop, void *dresidual_dev, int64_t ldr, void *dx_dev, int64_t ldx, float *dgamma_dev,
                             float *dbeta_dev)
{
    static const char *call = "leann_layernorm_backward";
    if (!ctx || !gamma_dev || !dgamma_dev || !dbeta_dev) {
        leann_set_error("%s: null context, scale or gradient of scale or shift", call);
        return LEANN_EINVAL;
    }
    LEANN_TRY(check_matrix(call, rows, cols, dtype));
    if (cols > MAX_COLS) {
        leann_set_error("%s: rows of %d elements are not covered (at most %d)", call, cols, MAX_COLS);
        return LEANN_ESHAPE;
    }
    Drop d;
    LEANN_TRY(make_drop(call, drop, &d));
    if (rows > 0) {
        LEANN_TRY(check_rows(call, "dout", dout_dev, ldd, cols));
        LEANN_TRY(check_rows(call, "total", total_dev, ldt, cols));
        if (dtotal_dev) LEANN_TRY(check_rows(call, "dtotal", dtotal_dev, lde, cols));
        LEANN_TRY(check_rows(call, "dresidual", dresidual_dev, ldr, cols));
        if (d.below) LEANN_TRY(check_rows(call, "dx", dx_dev, ldx, cols));
        if (!mean_dev || !rstd_dev) {
            leann_set_error("%s: mean or rstd is null", call);
            return LEANN_EINVAL;
        }
    }
    LEANN_HIP(hipSetDevice(ctx->device));
    std::lock_guard<std::mutex> turn(ctx->op_work_mutex);
    return with_type(dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        return with_row_shape(cols, [&](auto lpr, auto nc) {
            constexpr int LPR = decltype(lpr)::value, NC = decltype(nc)::value;
            const int64_t wanted = (rows + 256 / LPR - 1) / (256 / LPR);
            const unsigned grid = (unsigned)std::min<int64_t>(wanted, (int64_t)ctx->num_cus * 2);
            LEANN_TRY(ctx->reserve(ctx->op_work, std::max<size_t>(1, (size_t)grid * 2 * cols * sizeof(float))));
            float *partial = (float *)ctx->op_work.p;
            if (grid) {
                auto go = [&](auto kernel) {
                    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), LPR <= 64 ? NC * LPR * 8 * 2 * sizeof(float) : 0,
                                       ctx->stream, (const T *)dout_dev, ldd, (const T *)total_dev, ldt, (int)rows, (int)cols, gamma_dev, mean_dev,
                                       rstd_dev, (const T *)dtotal_dev, lde, (T *)dresidual_dev, ldr, (T *)dx_dev, ldx, partial, streams(rows, cols, sizeof(T)), d);
                };
                if (d.below) go(layernorm_grad_kernel<T, LPR, NC, true>);
                else go(layernorm_grad_kernel<T, LPR, NC, false>);
            }
            hipLaunchKernelGGL(column_sum_kernel, dim3((2 * cols + 15) / 16), dim3(1024), 0, ctx->stream, partial, (int)grid, (int)cols, dgamma_dev,
                               dbeta_dev);
            return launched(call);
        });
    });
}

}  // extern "C"
