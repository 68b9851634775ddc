// GELU with its gradient, and activations kept in 8 bits between the forward and the backward pass (gfx950).
#include <algorithm>

#include "row_calls.h"
#include "wave.h"

namespace {

// A checkpoint: of each row's 128 columns, a = max |x|, scale = a / 127, code = 127 x / a to the nearest whole number, ties to even; it stands for code * scale, off by at most
// half a scale.  16 lanes have 128 columns, eight elements each, and find a by register moves.  An infinity makes the scale infinite and all codes 0, a NaN makes the scale NaN,
// whatever the codes: all 128 come back as NaN.
// All kernels here are one pass, bound by memory; a thread has UNITS accesses on their way.  131072 x 768 bf16: kept in 55 us, back in 46 (5.6 TB/s); x 1536: GELU with its input kept
// 222 us (4.6 TB/s, as much as a copy), the gradient with the output once more 303 (4.6).
constexpr int BLOCK = 128;
constexpr int UNITS = 4;

enum { NO_ACTIVATION = -1 };

// Which rows and 128 columns a group of 16 lanes takes: every `step`-th.
struct Units {
    int64_t row, row_step;
    int blk, blk_step, blocks;
    __device__ inline Units(int cols)
    {
        blocks = (cols + BLOCK - 1) / BLOCK;
        const uint32_t first = blockIdx.x * 16 + (threadIdx.x >> 4), step = gridDim.x * 16;
        row = first / (uint32_t)blocks;
        blk = (int)(first % (uint32_t)blocks);
        row_step = step / (uint32_t)blocks;
        blk_step = (int)(step % (uint32_t)blocks);
    }
    __device__ inline void advance()
    {
        row += row_step;
        blk += blk_step;
        if (blk >= blocks) {
            blk -= blocks;
            ++row;
        }
    }
};

// One of UNITS: where it lies, and how many of the lane's eight columns there are (0: none, or no such row).
struct Place {
    int64_t row;
    int blk, n;
    __device__ inline int col() const { return blk * BLOCK + (threadIdx.x & 15) * 8; }
};
__device__ inline Place place(Units &u, int rows, int cols)
{
    Place p = {u.row, u.blk, 0};
    if (u.row < rows) p.n = max(0, min(8, cols - p.col()));
    u.advance();
    return p;
}

__device__ inline uint32_t max16(uint32_t v)  // over the 16 lanes of a row of lanes
{
    v = max(v, dpp_mov<DPP_ROW_ROR8>(v));
    v = max(v, dpp_mov<DPP_ROW_ROR4>(v));
    v = max(v, dpp_mov<DPP_ROW_ROR2>(v));
    return max(v, dpp_mov<DPP_QUAD_XOR1>(v));
}

// Phi(x), or its tanh form, and where GRAD is the derivative of x Phi(x).  Phi by 7.1.26 of Abramowitz and Stegun (Handbook of Mathematical Functions), whose erfc is off by at most
// 1.5e-7 and whose exponential is the derivative's, too: of Phi itself 0.16 % at -5, 0.4 % (a half step of bf16) at -6, 3 % at -12; the other by (1 + tanh u) / 2 = 1 / (1 + e^(-2u)).
template <int KIND, bool GRAD>
__device__ inline float distribution(float x, float &slope)
{
    if constexpr (KIND == LEANN_GELU) {
        const float e = __builtin_amdgcn_exp2f(x * x * -0.72134752f);  // e^(-x^2 / 2)
        const float t = __builtin_amdgcn_rcpf(fmaf(__builtin_fabsf(x), 0.23164189f, 1.f));
        float p = fmaf(t, 0.53070271f, -0.72657601f);  // half of the published coefficients: erfc / 2
        p = fmaf(t, p, 0.71070687f);
        p = fmaf(t, p, -0.14224837f);
        p = fmaf(t, p, 0.12741479f);
        const float tail = p * t * e, phi = x > 0.f ? 1.f - tail : tail;
        if constexpr (GRAD) slope = fmaf(x * 0.39894228f, e, phi);
        return x == x ? phi : x;
    } else {
        const float x2 = __builtin_fminf(x * x, 1e30f);
        const float g = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * fmaf(x2, -0.10294324f, -2.3022082f)));  // 2 sqrt(2 / pi) log2 e, and that times 0.044715
        if constexpr (GRAD) slope = fmaf(x * (g - g * g), fmaf(x2, 0.21406445f, 1.5957691f), g);
        return g;
    }
}

// codes and, in one lane of 16, the scale of a lane's eight elements (those behind the row's end are 0).
template <class T>
__device__ inline uint2 encode(const f32x8 &x, float &scale)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);  // as whole numbers NaN is the largest
    const float a = __uint_as_float(max16(most));
    scale = a / 127.f;
    // out of the way of overflows, of 127 x and of the reciprocal
    const float k = a > 0x1p60f ? 0x1p-60f : a < 0x1p-60f ? 0x1p60f : 1.f, b = a > 0.f ? a * k : 1.f;
    const float r = __builtin_amdgcn_rcpf(b);
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = x[i] * k * 127.f;
        float c;
        if constexpr (sizeof(T) == 4) {
            c = y / b;
        } else {
            // 16-bit numbers: a quotient that is no tie is 2^-19 of itself away from one, more than this is off; one step of refinement makes ties exact
            c = y * r;
            c = fmaf(fmaf(-c, b, y), r, c);
        }
        q[i] = __float_as_uint(c + 0x1.8p23f);  // the nearest whole number in the low bits, of NaN 0
    }
    auto four = [](const uint32_t *v) {
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(v[3], v[2], 0x0c0c0400), __builtin_amdgcn_perm(v[1], v[0], 0x0c0c0400), 0x05040100);
    };
    return make_uint2(four(q), four(q + 4));
}

__device__ inline f32x8 decode(const uint2 &codes, float scale)
{
    f32x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)((i < 4 ? codes.x : codes.y) >> (8 * (i & 3))) * scale;
    return x;
}

struct Codes8 {
    uint2 v;
    __device__ inline void load(const int8_t *p, int n)
    {
        if (n >= 8) {
            __builtin_memcpy(&v, p, 8);
        } else {
            uint32_t w[2] = {0, 0};
            for (int i = 0; i < n; ++i) w[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
            v = make_uint2(w[0], w[1]);
        }
    }
    __device__ inline void store(int8_t *p, int n) const
    {
        if (n >= 8) {
            __builtin_memcpy(p, &v, 8);
        } else {
            for (int i = 0; i < n; ++i) p[i] = (int8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
        }
    }
};

// out = x Phi(x), unless KIND is NO_ACTIVATION; with KEEP, x in 8 bits.
template <class T, int KIND, bool KEEP>
__global__ __launch_bounds__(256) void activate_kernel(const T *x, int64_t ldx, int rows, int cols, T *out, int64_t ldo, int8_t *codes, int64_t ldc, float *scales,
                                                       int streaming)
{
    Units units(cols);
    while (units.row < rows) {
        Place p[UNITS];
        Raw8<T> v[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            p[i] = place(units, rows, cols);
            v[i].load(x + p[i].row * ldx + p[i].col(), p[i].n);
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const f32x8 w = v[i].wide();
            if constexpr (KEEP) {
                float scale;
                Codes8 c;
                c.v = encode<T>(w, scale);
                if (p[i].n > 0) {
                    c.store(codes + p[i].row * ldc + p[i].col(), p[i].n);
                    if ((threadIdx.x & 15) == 0) scales[p[i].row * units.blocks + p[i].blk] = scale;
                }
            }
            if constexpr (KIND != NO_ACTIVATION) {
                f32x8 y;
                float none;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = w[e] * distribution<KIND, false>(w[e], none);
                v[i].round(y);
                if (p[i].n > 0) v[i].store(out + p[i].row * ldo + p[i].col(), p[i].n, streaming);
            }
        }
    }
}

// x again from 8 bits.
template <class T>
__global__ __launch_bounds__(256) void restore_kernel(const int8_t *codes, int64_t ldc, const float *scales, int rows, int cols, T *out, int64_t ldo, int streaming)
{
    Units units(cols);
    while (units.row < rows) {
        Place p[UNITS];
        Codes8 c[UNITS];
        float scale[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            p[i] = place(units, rows, cols);
            c[i].load(codes + p[i].row * ldc + p[i].col(), p[i].n);
            scale[i] = p[i].n > 0 ? scales[p[i].row * units.blocks + p[i].blk] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            Raw8<T> v;
            v.round(decode(c[i].v, scale[i]));
            if (p[i].n > 0) v.store(out + p[i].row * ldo + p[i].col(), p[i].n, streaming);
        }
    }
}

// dx = dout (x Phi(x))', x from 8 bits or as it was; with AGAIN x Phi(x), too.
template <class T, int KIND, bool KEPT, bool AGAIN>
__global__ __launch_bounds__(256) void activation_grad_kernel(const T *dout, int64_t ldd, const T *x, int64_t ldx, const int8_t *codes, int64_t ldc, const float *scales, int rows,
                                                              int cols, T *dx, int64_t lddx, T *again, int64_t lda, int streaming)
{
    Units units(cols);
    while (units.row < rows) {
        Place p[UNITS];
        Raw8<T> g[UNITS], v[UNITS];
        Codes8 c[UNITS];
        float scale[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            p[i] = place(units, rows, cols);
            g[i].load(dout + p[i].row * ldd + p[i].col(), p[i].n);
            if constexpr (KEPT) {
                c[i].load(codes + p[i].row * ldc + p[i].col(), p[i].n);
                scale[i] = p[i].n > 0 ? scales[p[i].row * units.blocks + p[i].blk] : 0.f;
            } else {
                v[i].load(x + p[i].row * ldx + p[i].col(), p[i].n);
            }
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const f32x8 w = KEPT ? decode(c[i].v, scale[i]) : v[i].wide(), dy = g[i].wide();
            f32x8 y, d;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float slope;
                y[e] = w[e] * distribution<KIND, true>(w[e], slope);
                d[e] = dy[e] * slope;
            }
            g[i].round(d);
            v[i].round(y);
            if (p[i].n > 0) {
                g[i].store(dx + p[i].row * lddx + p[i].col(), p[i].n, streaming);
                if constexpr (AGAIN) v[i].store(again + p[i].row * lda + p[i].col(), p[i].n, streaming);
            }
        }
    }
}

int check_call(const char *call, const leann_ctx *ctx, int64_t rows, int64_t cols, int dtype, int kind)
{
    if (!ctx || (kind != LEANN_GELU && kind != LEANN_GELU_TANH && kind != NO_ACTIVATION)) {
        leann_set_error("%s: null context or unknown activation", call);
        return LEANN_EINVAL;
    }
    LEANN_TRY(check_matrix(call, rows, cols, dtype));
    if (rows * ((cols + BLOCK - 1) / BLOCK) > 0xffffffffll - 0x1000000) {  // numbers of 128 columns, and a step further, are 32 bits
        leann_set_error("%s: %lld rows of %lld 128 columns are not covered (below 2^32 - 2^24 together)", call, (long long)rows, (long long)((cols + BLOCK - 1) / BLOCK));
        return LEANN_ESHAPE;
    }
    return LEANN_OK;
}

int check_kept(const char *call, const int8_t *codes, int64_t ldc, const float *scales, int64_t cols)
{
    LEANN_TRY(check_rows(call, "codes", codes, ldc, cols));
    if (!scales) {
        leann_set_error("%s: scales is null", call);
        return LEANN_EINVAL;
    }
    return LEANN_OK;
}

unsigned grid_of(const leann_ctx *ctx, int64_t rows, int64_t cols)
{
    const int64_t units = rows * ((cols + BLOCK - 1) / BLOCK);
    return (unsigned)std::min<int64_t>((units + 15) / 16, (int64_t)ctx->num_cus * 8);
}

int activate(const char *call, leann_ctx *ctx, const void *x_dev, int64_t ldx, int64_t rows, int64_t cols, int dtype, int kind, void *out_dev, int64_t ldo, int8_t *codes_dev,
             int64_t ldc, float *scales_dev)
{
    LEANN_HIP(hipSetDevice(ctx->device));
    return with_type(dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(grid_of(ctx, rows, cols)), dim3(256), 0, ctx->stream, (const T *)x_dev, ldx, (int)rows, (int)cols, (T *)out_dev, ldo, codes_dev, ldc,
                               scales_dev, streams(rows, cols, sizeof(T)));
        };
        if (kind == NO_ACTIVATION) go(activate_kernel<T, NO_ACTIVATION, true>);
        else if (kind == LEANN_GELU) codes_dev ? go(activate_kernel<T, LEANN_GELU, true>) : go(activate_kernel<T, LEANN_GELU, false>);
        else codes_dev ? go(activate_kernel<T, LEANN_GELU_TANH, true>) : go(activate_kernel<T, LEANN_GELU_TANH, false>);
        return launched(call);
    });
}

}  // namespace

extern "C" {

int leann_checkpoint(leann_ctx *ctx, const void *x_dev, int64_t ldx, int64_t rows, int64_t cols, int dtype, int8_t *codes_dev, int64_t ldc, float *scales_dev)
{
    static const char *call = "leann_checkpoint";
    LEANN_TRY(check_call(call, ctx, rows, cols, dtype, NO_ACTIVATION));
    if (rows == 0) return LEANN_OK;
    LEANN_TRY(check_rows(call, "x", x_dev, ldx, cols));
    LEANN_TRY(check_kept(call, codes_dev, ldc, scales_dev, cols));
    return activate(call, ctx, x_dev, ldx, rows, cols, dtype, NO_ACTIVATION, nullptr, 0, codes_dev, ldc, scales_dev);
}

int leann_checkpoint_restore(leann_ctx *ctx, const int8_t *codes_dev, int64_t ldc, const float *scales_dev, int64_t rows, int64_t cols, int dtype, void *out_dev, int64_t ldo)
{
    static const char *call = "leann_checkpoint_restore";
    LEANN_TRY(check_call(call, ctx, rows, cols, dtype, NO_ACTIVATION));
    if (rows == 0) return LEANN_OK;
    LEANN_TRY(check_kept(call, codes_dev, ldc, scales_dev, cols));
    LEANN_TRY(check_rows(call, "out", out_dev, ldo, cols));
    LEANN_HIP(hipSetDevice(ctx->device));
    return with_type(dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        hipLaunchKernelGGL(restore_kernel<T>, dim3(grid_of(ctx, rows, cols)), dim3(256), 0, ctx->stream, codes_dev, ldc, scales_dev, (int)rows, (int)cols, (T *)out_dev, ldo,
                           streams(rows, cols, sizeof(T)));
        return launched(call);
    });
}

int leann_activation(leann_ctx *ctx, const void *x_dev, int64_t ldx, int64_t rows, int64_t cols, int dtype, int kind, void *out_dev, int64_t ldo, int8_t *codes_dev, int64_t ldc,
                     float *scales_dev)
{
    static const char *call = "leann_activation";
    LEANN_TRY(check_call(call, ctx, rows, cols, dtype, kind));
    if (kind == NO_ACTIVATION || !codes_dev != !scales_dev) {
        leann_set_error("%s: unknown activation, or only one of codes and scales", call);
        return LEANN_EINVAL;
    }
    if (rows == 0) return LEANN_OK;
    LEANN_TRY(check_rows(call, "x", x_dev, ldx, cols));
    LEANN_TRY(check_rows(call, "out", out_dev, ldo, cols));
    if (codes_dev) LEANN_TRY(check_kept(call, codes_dev, ldc, scales_dev, cols));
    return activate(call, ctx, x_dev, ldx, rows, cols, dtype, kind, out_dev, ldo, codes_dev, ldc, scales_dev);
}

int leann_activation_backward(leann_ctx *ctx, const void *dout_dev, int64_t ldd, const void *x_dev, int64_t ldx, const int8_t *codes_dev, int64_t ldc, const float *scales_dev,
                              int64_t rows, int64_t cols, int dtype, int kind, void *dx_dev, int64_t lddx, void *again_dev, int64_t lda)
{
    static const char *call = "leann_activation_backward";
    LEANN_TRY(check_call(call, ctx, rows, cols, dtype, kind));
    if (kind == NO_ACTIVATION || (rows > 0 && !x_dev == !codes_dev)) {
        leann_set_error("%s: unknown activation, or x and codes both or neither", call);
        return LEANN_EINVAL;
    }
    if (rows == 0) return LEANN_OK;
    LEANN_TRY(check_rows(call, "dout", dout_dev, ldd, cols));
    LEANN_TRY(check_rows(call, "dx", dx_dev, lddx, cols));
    if (x_dev) LEANN_TRY(check_rows(call, "x", x_dev, ldx, cols));
    else LEANN_TRY(check_kept(call, codes_dev, ldc, scales_dev, cols));
    if (again_dev) LEANN_TRY(check_rows(call, "again", again_dev, lda, cols));
    LEANN_HIP(hipSetDevice(ctx->device));
    return with_type(dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        auto with_kind = [&](auto k) {
            constexpr int KIND = decltype(k)::value;
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3(grid_of(ctx, rows, cols)), dim3(256), 0, ctx->stream, (const T *)dout_dev, ldd, (const T *)x_dev, ldx, codes_dev, ldc, scales_dev,
                                   (int)rows, (int)cols, (T *)dx_dev, lddx, (T *)again_dev, lda, streams(rows, cols, sizeof(T)));
            };
            if (x_dev) again_dev ? go(activation_grad_kernel<T, KIND, false, true>) : go(activation_grad_kernel<T, KIND, false, false>);
            else again_dev ? go(activation_grad_kernel<T, KIND, true, true>) : go(activation_grad_kernel<T, KIND, true, false>);
        };
        if (kind == LEANN_GELU) with_kind(std::integral_constant<int, LEANN_GELU>());
        else with_kind(std::integral_constant<int, LEANN_GELU_TANH>());
        return launched(call);
    });
}

}  // extern "C"
