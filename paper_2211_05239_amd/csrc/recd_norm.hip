// Layer norm of rows [n, D] and its gradients.
//
//   h = (x - mean(x)) * rstd,  rstd = 1 / sqrt(mean((x - mean(x))^2) + eps),  y = h * w + b
//   with u = g * w:  gx = rstd * (u - mean(u) - h * mean(u * h)),  gw = sum over rows of g * h,  gb = sum of g
//
// Both directions are bound by HBM traffic: the forward pass reads a row and writes one, the backward pass reads
// two and writes one.  300 007 x 128 bf16: 33 us forward (154 MB, 4.7 TB/s, what a large copy reaches), 42 us backward (230 MB,
// 5.5 TB/s, part of it from the caches), and 5 us for the sums of the weight's and the bias's gradients.
// A row lives in the registers of 2^glog lanes, `P` pieces of 16 bytes in each, from its only read to its write: the variance is
// taken about the mean from the registers, in 32 bits, not from a sum of squares.
// The weight and the bias of a lane's columns stay in its registers over all rows that the lane group takes.
// The sums over the rows: every lane adds up its columns over its group's rows, a block adds up its groups (lane
// exchanges, then LDS), and a second launch adds up the blocks' rows of partial sums in their order, so the
// result depends on the sizes alone.
#include "recd_internal.h"
#include "recd_vec.h"

namespace {

constexpr int kBlock = 256;

__device__ inline float group_sum(float v, int glog)
{
    for (int o = (1 << glog) >> 1; o; o >>= 1)
        v += __shfl_xor(v, o);
    return v;
}

template <typename T, int P>
__global__ __launch_bounds__(kBlock) void k_layer_norm(int64_t n, int D, int glog, const T *x,  // (may be y)
                                                       const float *__restrict__ weight, const float *__restrict__ bias,
                                                       float eps, T *y, float2 *stats)
{
    constexpr int E = 16 / sizeof(T);
    const int vecs = D / E, G = 1 << glog, lane = threadIdx.x & (G - 1);
    const int64_t groups = (int64_t)gridDim.x * (kBlock >> glog);
    const float inv = 1.0f / (float)D;
    float w[P * E], b[P * E];
    bool in[P];
    for (int p = 0; p < P; p++) {
        const int v = lane + p * G;
        in[p] = v < vecs;
        for (int e = 0; e < E; e++) {
            w[p * E + e] = in[p] && weight ? weight[v * E + e] : 1.0f;
            b[p * E + e] = in[p] && bias ? bias[v * E + e] : 0.0f;
        }
    }
    for (int64_t r = (int64_t)blockIdx.x * (kBlock >> glog) + (threadIdx.x >> glog); r < n; r += groups) {
        float a[P * E];
        float s = 0.0f;
        for (int p = 0; p < P; p++) {
            if (in[p])
                recd_load16(x + r * D + (lane + p * G) * E, a + p * E);
            for (int e = 0; e < E; e++) {
                a[p * E + e] = in[p] ? a[p * E + e] : 0.0f;
                s += a[p * E + e];
            }
        }
        const float mean = group_sum(s, glog) * inv;
        float q = 0.0f;
        for (int p = 0; p < P; p++)
            for (int e = 0; e < E; e++) {
                a[p * E + e] = in[p] ? a[p * E + e] - mean : 0.0f;
                q += a[p * E + e] * a[p * E + e];
            }
        const float rstd = 1.0f / sqrtf(group_sum(q, glog) * inv + eps);
        for (int p = 0; p < P; p++)
            if (in[p]) {
                for (int e = 0; e < E; e++)
                    a[p * E + e] = a[p * E + e] * rstd * w[p * E + e] + b[p * E + e];
                recd_store16(y + r * D + (lane + p * G) * E, a + p * E);
            }
        if (stats && lane == 0)
            stats[r] = make_float2(mean, rstd);
    }
}

// part: [gridDim.x][2][D], the block's sums of g * h and of g
template <typename T, int P>
__global__ __launch_bounds__(kBlock) void k_layer_norm_backward(int64_t n, int D, int glog, const T *__restrict__ x,
                                                                const float *__restrict__ weight,
                                                                const float2 *__restrict__ stats, const T *grad_y,
                                                                T *grad_x, float *__restrict__ part)
{
    constexpr int E = 16 / sizeof(T);
    extern __shared__ float sums[];  // [waves - 1][2][D]
    const int vecs = D / E, G = 1 << glog, lane = threadIdx.x & (G - 1);
    const int64_t groups = (int64_t)gridDim.x * (kBlock >> glog);
    const float inv = 1.0f / (float)D;
    float w[P * E], gw[P * E], gb[P * E];
    bool in[P];
    for (int p = 0; p < P; p++) {
        const int v = lane + p * G;
        in[p] = v < vecs;
        for (int e = 0; e < E; e++) {
            w[p * E + e] = in[p] && weight ? weight[v * E + e] : 1.0f;
            gw[p * E + e] = gb[p * E + e] = 0.0f;
        }
    }
    for (int64_t r = (int64_t)blockIdx.x * (kBlock >> glog) + (threadIdx.x >> glog); r < n; r += groups) {
        const float2 st = stats[r];
        float h[P * E], g[P * E];
        float s1 = 0.0f, s2 = 0.0f;
        for (int p = 0; p < P; p++) {
            const int64_t at = r * D + (lane + p * G) * E;
            if (in[p]) {
                recd_load16(x + at, h + p * E);
                recd_load16(grad_y + at, g + p * E);
            }
            for (int e = 0; e < E; e++) {
                const int i = p * E + e;
                h[i] = in[p] ? (h[i] - st.x) * st.y : 0.0f;
                g[i] = in[p] ? g[i] : 0.0f;
                gw[i] += g[i] * h[i];
                gb[i] += g[i];
                g[i] *= w[i];
                s1 += g[i];
                s2 += g[i] * h[i];
            }
        }
        s1 = group_sum(s1, glog) * inv;
        s2 = group_sum(s2, glog) * inv;
        for (int p = 0; p < P; p++)
            if (in[p]) {
                for (int e = 0; e < E; e++)
                    g[p * E + e] = st.y * (g[p * E + e] - s1 - h[p * E + e] * s2);
                recd_store16(grad_x + r * D + (lane + p * G) * E, g + p * E);
            }
    }
    if (!part)
        return;
    for (int i = 0; i < P * E; i++)
        for (int o = G; o < 64; o <<= 1) {
            gw[i] += __shfl_xor(gw[i], o);
            gb[i] += __shfl_xor(gb[i], o);
        }
    const int wave = threadIdx.x >> 6;
    const bool holds = (threadIdx.x & 63) < G;
    if (wave && holds)
        for (int p = 0; p < P; p++)
            if (in[p])
                for (int e = 0; e < E; e++) {
                    sums[(wave - 1) * 2 * D + (lane + p * G) * E + e] = gw[p * E + e];
                    sums[(wave - 1) * 2 * D + D + (lane + p * G) * E + e] = gb[p * E + e];
                }
    __syncthreads();
    if (wave == 0 && holds)
        for (int p = 0; p < P; p++)
            if (in[p])
                for (int e = 0; e < E; e++) {
                    const int col = (lane + p * G) * E + e;
                    float a = gw[p * E + e], b = gb[p * E + e];
                    for (int k = 0; k < kBlock / 64 - 1; k++) {
                        a += sums[k * 2 * D + col];
                        b += sums[k * 2 * D + D + col];
                    }
                    part[(int64_t)blockIdx.x * 2 * D + col] = a;
                    part[(int64_t)blockIdx.x * 2 * D + D + col] = b;
                }
}

// Columns of the blocks' partial sums: 32 columns by 32 rows of threads, rows in steps of 32, then the rows' sums.
__global__ __launch_bounds__(1024) void k_sum_parts(int blocks, int D, const float *__restrict__ part, float *grad_weight,
                                                    float *grad_bias)
{
    __shared__ float rows[32][33];
    const int c = threadIdx.x & 31, row = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    float s = 0.0f;
    if (col < 2 * D)
#pragma unroll 8
        for (int i = row; i < blocks; i += 32)
            s += part[(int64_t)i * 2 * D + col];
    rows[row][c] = s;
    __syncthreads();
    if (row)
        return;
    s = 0.0f;
    for (int i = 0; i < 32; i++)
        s += rows[i][c];
    if (col < D && grad_weight)
        grad_weight[col] = s;
    if (col >= D && col < 2 * D && grad_bias)
        grad_bias[col - D] = s;
}

// Lanes and pieces of a row: as few idle lanes as possible, and of equal ones the fewest pieces a lane. With two pieces a lane
// where one would do, forward and backward of 300 007 rows of 64 bf16 take 63 us against 48, of 128 elements 101 against 92;
// with four, 134 and 164 (at eight blocks a compute unit).
struct Shape {
    int P, glog;
};

Shape row_shape(int vecs)
{
    Shape best{0, 0};
    int cost = 1 << 30;
    for (int P : {1, 2, 3, 4}) {
        int glog = 0;
        while ((P << glog) < vecs)
            glog++;
        if (glog <= 6 && (P << glog) < cost) {
            cost = P << glog;
            best = {P, glog};
        }
    }
    return best;
}

recd_status check_norm(recd_ctx *ctx, int64_t n, int D, recd_dtype dt)
{
    if (!ctx)
        return RECD_EINVAL;
    if (n < 0)
        return recd_fail(ctx, RECD_EINVAL, "n < 0");
    if ((int)dt < 0 || (int)dt > 2)
        return recd_fail(ctx, RECD_EINVAL, "unknown dtype");
    const int64_t rb = (int64_t)D * (int64_t)elem_size(dt);
    if (D <= 0 || rb % 16 != 0 || rb > RECD_MAX_ROW_BYTES)
        return recd_fail(ctx, RECD_EINVAL, "D=%d: row bytes %lld must be a multiple of 16 and <= %d", D, (long long)rb,
                         RECD_MAX_ROW_BYTES);
    return RECD_OK;
}

// Blocks of a launch: four a compute unit, whose lanes read the weight once.  Forward and backward of 300 007 x 128 bf16 with
// two, four, eight and sixteen: 115, 88, 97 and 109 us; 50 021 x 516 fp32 132, 101, 110 and 117; forward alone 45, 33, 34.
int64_t norm_blocks(const recd_ctx *ctx, int64_t n, int glog)
{
    const int64_t need = (n + (kBlock >> glog) - 1) / (kBlock >> glog);
    const int64_t most = (int64_t)ctx->num_cu * 4;
    return need < most ? need : most;
}

template <typename T, typename F> void with_pieces(int P, F f)
{
    switch (P) {
    case 1: f(std::integral_constant<int, 1>{}); break;
    case 2: f(std::integral_constant<int, 2>{}); break;
    case 3: f(std::integral_constant<int, 3>{}); break;
    default: f(std::integral_constant<int, 4>{}); break;
    }
}

size_t sums_bytes(const recd_ctx *ctx, int64_t n, int D, recd_dtype dt)
{
    return (size_t)norm_blocks(ctx, n, row_shape(D * (int)elem_size(dt) / 16).glog) * 2 * D * 4;
}

} // namespace

extern "C" {

recd_status recd_layer_norm_workspace_bytes(int device, int64_t n, int D, recd_dtype dt, size_t *out_bytes)
{
    recd_ctx c;
    if (!out_bytes)
        return RECD_EINVAL;
    RECD_TRY(check_norm(&c, n, D, dt));
    RECD_TRY(recd_sizing_context(&c, device));
    *out_bytes = sums_bytes(&c, n, D, dt);
    return RECD_OK;
}

recd_status recd_layer_norm(recd_ctx *ctx, int64_t n, int D, recd_dtype dt, const void *x, const float *weight,
                            const float *bias, float eps, void *y, float *stats)
{
    RECD_TRY(check_norm(ctx, n, D, dt));
    if (n == 0)
        return RECD_OK;
    if (!x || !y)
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (((uintptr_t)x | (uintptr_t)y) % 16 || (uintptr_t)stats % 8)
        return recd_fail(ctx, RECD_EINVAL, "x and y must be aligned to 16 bytes, stats to 8");
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    const Shape s = row_shape(D * (int)elem_size(dt) / 16);
    const dim3 grid((unsigned)norm_blocks(ctx, n, s.glog));
    recd_with_type(dt, [&](auto t) {
        using T = decltype(t);
        with_pieces<T>(s.P, [&](auto p) {
            hipLaunchKernelGGL((k_layer_norm<T, p.value>), grid, dim3(kBlock), 0, ctx->stream, n, D, s.glog, (const T *)x,
                               weight, bias, eps, (T *)y, (float2 *)stats);
        });
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

recd_status recd_layer_norm_backward(recd_ctx *ctx, int64_t n, int D, recd_dtype dt, const void *x, const float *weight,
                                     const float *stats, const void *grad_y, void *grad_x, float *grad_weight,
                                     float *grad_bias)
{
    RECD_TRY(check_norm(ctx, n, D, dt));
    if (n > 0 && (!x || !stats || !grad_y || !grad_x))
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (((uintptr_t)x | (uintptr_t)grad_y | (uintptr_t)grad_x) % 16 || (uintptr_t)stats % 8)
        return recd_fail(ctx, RECD_EINVAL, "x, grad_y and grad_x must be aligned to 16 bytes, stats to 8");
    const bool sums = grad_weight || grad_bias;
    if (n == 0 && !sums)
        return RECD_OK;
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    const Shape s = row_shape(D * (int)elem_size(dt) / 16);
    const int64_t blocks = norm_blocks(ctx, n, s.glog);
    float *part = nullptr;
    if (sums) {
        ctx->plan.valid = false;  // the partial sums overwrite the workspace a backward plan would live in
        RECD_TRY(recd_reserve(ctx, sums_bytes(ctx, n, D, dt)));
        part = reinterpret_cast<float *>(ctx->ws);
    }
    if (n > 0)
        recd_with_type(dt, [&](auto t) {
            using T = decltype(t);
            with_pieces<T>(s.P, [&](auto p) {
                hipLaunchKernelGGL((k_layer_norm_backward<T, p.value>), dim3((unsigned)blocks), dim3(kBlock),
                                   sums ? (kBlock / 64 - 1) * 2 * D * 4 : 0, ctx->stream, n, D, s.glog, (const T *)x, weight,
                                   (const float2 *)stats, (const T *)grad_y, (T *)grad_x, part);
            });
        });
    if (sums)
        hipLaunchKernelGGL(k_sum_parts, dim3((unsigned)((2 * D + 31) / 32)), dim3(1024), 0, ctx->stream, (int)blocks, D, part,
                           grad_weight, grad_bias);
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

} // extern "C"
