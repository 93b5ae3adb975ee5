// Dropout of rows [n, D] behind a residual, and its gradient.
//
//   out = residual + x * mask / (1 - p),  grad_x = grad_out * mask / (1 - p)
//
// Bound by HBM traffic: a row of each operand is read and one written.  300 007 x 128 bf16, both directions (384 MB, part of it in
// the caches): 76 us, 5.05 TB/s, what a large copy reaches; 50 021 x 516 fp32 79 us.  A thread goes through pieces of 16 bytes, kPieces of
// which are read before the first is worked on; the next piece's row and column follow by additions, without a division.
#include "recd_epilogue.h"

#include <math.h>

namespace {

constexpr int kBlock = 256, kPieces = 4;

// A lane takes 16 bytes of a row at a time: eight 16-bit elements, or four 32-bit ones, whose neighbouring lane has the other half
// of the mask's piece (and makes its bits again: lanes of eight elements each, 32 bytes apart, ask for half lines, 96 us in place of 79 for
// both directions of 50 021 x 516).
template <typename T, bool RES>
__global__ __launch_bounds__(kBlock) void k_dropout(int64_t pieces, int per_row, int D, RecdMask mask, const T *x,  // (may be out)
                                                    const T *res, T *out)
{
    constexpr int E = 16 / sizeof(T);
    using Piece = typename RecdPiece<T>::type;
    const int64_t threads = (int64_t)gridDim.x * kBlock;
    // piece `at` is piece `col` of row `row`; on by `threads` pieces: `drow` rows and `dcol` pieces
    int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    int64_t row = at / per_row;
    int col = (int)(at - row * per_row);
    const int64_t drow = threads / per_row;
    const int dcol = (int)(threads - drow * per_row);
    const uint64_t call = recd_mask_call(mask);
    while (at < pieces) {
        Piece v[kPieces], r[kPieces];
        int64_t rows[kPieces];
        int cols[kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
            rows[i] = row;
            cols[i] = col;
            if (at + i * threads < pieces) {
                const int64_t first = row * D + col * E;
                v[i] = *reinterpret_cast<const Piece *>(x + first);
                if constexpr (RES)
                    r[i] = *reinterpret_cast<const Piece *>(res + first);
            }
            row += drow;
            col += dcol;
            if (col >= per_row) {
                col -= per_row;
                row++;
            }
        }
#pragma unroll
        for (int i = 0; i < kPieces; i++)
            if (at + i * threads < pieces) {
                float y[E];
#pragma unroll
                for (int e = 0; e < E; e++)
                    y[e] = (float)v[i][e];
                if (mask.cut) {
                    RecdBits bits = recd_mask_bits(mask, call, rows[i], cols[i] * E / 8);
                    if constexpr (E == 4) {
                        bits.w[0] = cols[i] & 1 ? bits.w[2] : bits.w[0];
                        bits.w[1] = cols[i] & 1 ? bits.w[3] : bits.w[1];
                    }
#pragma unroll
                    for (int e = 0; e < E; e++)
                        y[e] = bits.keep(e, mask.cut) ? y[e] * mask.by : 0.0f;
                }
                Piece w;
#pragma unroll
                for (int e = 0; e < E; e++)
                    w[e] = (T)(RES ? y[e] + (float)r[i][e] : y[e]);
                __builtin_nontemporal_store(w, reinterpret_cast<Piece *>(out + rows[i] * D + cols[i] * E));
            }
        at += kPieces * threads;
    }
}

recd_status dropout(recd_ctx *ctx, int64_t n, int D, recd_dtype dt, const recd_dropout_mask *m, const void *x, const void *res,
                    void *out)
{
    if (!ctx)
        return RECD_EINVAL;
    if (n < 0 || n >= (int64_t)1 << 48)
        return recd_fail(ctx, RECD_EINVAL, "n=%lld outside [0, 2^48)", (long long)n);
    if ((int)dt < 0 || (int)dt > 2)
        return recd_fail(ctx, RECD_EINVAL, "unknown dtype");
    if (D <= 0 || D > RECD_MAX_WIDTH || D * elem_size(dt) % 16 != 0)
        return recd_fail(ctx, RECD_EINVAL, "D=%d: row bytes must be a multiple of 16, and D at most %d", D, RECD_MAX_WIDTH);
    if (!m)
        return recd_fail(ctx, RECD_EINVAL, "no mask");
    RecdMask mask;
    RECD_TRY(recd_make_mask(ctx, m, &mask));
    if (n == 0)
        return RECD_OK;
    if (!x || !out)
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (((uintptr_t)x | (uintptr_t)res | (uintptr_t)out) % 16)
        return recd_fail(ctx, RECD_EINVAL, "rows must be aligned to 16 bytes");
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    const int per_row = D * (int)elem_size(dt) / 16;
    const int64_t pieces = n * per_row, need = (pieces + kBlock - 1) / kBlock, most = (int64_t)ctx->num_cu * 8;
    const dim3 grid((unsigned)(need < most ? need : most));
    recd_with_type(dt, [&](auto t) {
        using T = decltype(t);
        if (res)
            hipLaunchKernelGGL((k_dropout<T, true>), grid, dim3(kBlock), 0, ctx->stream, pieces, per_row, D, mask, (const T *)x,
                               (const T *)res, (T *)out);
        else
            hipLaunchKernelGGL((k_dropout<T, false>), grid, dim3(kBlock), 0, ctx->stream, pieces, per_row, D, mask, (const T *)x,
                               (const T *)nullptr, (T *)out);
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

} // namespace

recd_status recd_make_mask(recd_ctx *ctx, const recd_dropout_mask *m, RecdMask *out)
{
    *out = RecdMask{0, 0, 0, 1.0f, 0, nullptr};
    if (!m)
        return RECD_OK;
    const double cut = floor(m->p * 65536.0 + 0.5);
    if (!(m->p >= 0.0) || !(cut < 65536.0))
        return recd_fail(ctx, RECD_EINVAL, "p=%g outside [0, 1), to 2^-16", m->p);
    if ((uintptr_t)m->step % 8)
        return recd_fail(ctx, RECD_EINVAL, "step must be aligned to 8 bytes");
    *out = RecdMask{(uint32_t)m->seed, (uint32_t)(m->seed >> 32), (uint32_t)cut, (float)(65536.0 / (65536.0 - cut)), m->call, m->step};
    return RECD_OK;
}

extern "C" {

recd_status recd_dropout(recd_ctx *ctx, int64_t n, int D, recd_dtype dt, const recd_dropout_mask *mask, const void *x,
                         const void *residual, void *out)
{
    return dropout(ctx, n, D, dt, mask, x, residual, out);
}

recd_status recd_dropout_backward(recd_ctx *ctx, int64_t n, int D, recd_dtype dt, const recd_dropout_mask *mask, const void *grad_out,
                                  void *grad_x)
{
    return dropout(ctx, n, D, dt, mask, grad_out, nullptr, grad_x);
}

} // extern "C"
