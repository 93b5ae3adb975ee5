// A dense layer on rows x [n, in] with weights w [out, in], and its gradients.
//
//   z = x w^T + bias,  y = residual + dropout(act(z))
//   gz = dropout'(grad_y) act'(z),  grad_x = gz w,  grad_w = gz^T x,  grad_bias = sum over rows of gz
//
// Every product is C[i, j] = sum over k of P[i, k] Q[j, k], either with both operands' rows along k (the layer itself and, with w
// transposed into the workspace, grad_x), or with both along i and j (grad_w, which sums over the rows).  Blocks stage
// tiles of both through registers into two buffers of LDS; a wave multiplies TI x TJ tiles of 32 x 32 on the matrix cores, features
// as the product's rows and rows of x as its columns, so that a lane ends up with four neighbouring features of one row.  The sums go
// through LDS once more: bias, activation, dropout, residual and the store work on eight neighbouring features a lane.
#include "recd_epilogue.h"
#include "recd_mfma.h"

#include <math.h>

namespace {

constexpr int kBlock = 256;

enum { FORWARD = 0, GRAD = 1, PLAIN = 2 };

// What becomes of the sums.  Strides in bytes.
struct Epilogue {
    int act;
    RecdMask mask;
    int64_t row0;          // the first row's number, for the mask
    const float *bias;
    const void *other;     // FORWARD: residual, GRAD: grad_y
    int64_t other_stride;
    void *out;             // FORWARD: y, GRAD: gz (or null), PLAIN: the product
    int64_t out_stride;
    float *sums;           // FORWARD: receives z [n_i, n_j], or null
    float *col_part;       // GRAD: sums of gz over the rows of a block, [blocks][n_j], or null
};

struct ProductArgs {
    int64_t n_i;
    int n_j;
    int64_t K, k_each;     // contraction, and what one split takes of it
    const void *p, *q;
    int64_t p_stride, q_stride;  // bytes
    int tiles_i, tiles_j, splits;
    float *part;           // with several splits: their sums [splits][n_i][n_j]
    Epilogue e;
};

// Eight (`count`) sums of row `row` from column `col` on.  `b`: the columns' bias.
template <typename T, int KIND>
__device__ inline void finish(const Epilogue &e, uint64_t call, int64_t row, int col, int count, int n_j, const float *b, float *z,
                              float *col_sum)
{
    float v[8];
    if constexpr (KIND == FORWARD) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            v[i] = z[i] + b[i];
        if (e.sums)
            recd_store8(e.sums + row * n_j + col, count, v);
        recd_activate(e.act, v);
        if (e.mask.cut)
            recd_mask_apply(e.mask, recd_mask_bits(e.mask, call, e.row0 + row, col >> 3), v);
        if (e.other) {
            float r[8];
            recd_load8(reinterpret_cast<const T *>(reinterpret_cast<const char *>(e.other) + row * e.other_stride) + col, count, r);
#pragma unroll
            for (int i = 0; i < 8; i++)
                v[i] += r[i];
        }
    } else if constexpr (KIND == GRAD) {
        recd_load8(reinterpret_cast<const T *>(reinterpret_cast<const char *>(e.other) + row * e.other_stride) + col, count, v);
        if (e.mask.cut)
            recd_mask_apply(e.mask, recd_mask_bits(e.mask, call, e.row0 + row, col >> 3), v);
        if (e.act != RECD_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                z[i] += b[i];
            recd_activate_back(e.act, z, v);
        }
#pragma unroll
        for (int i = 0; i < 8; i++)
            col_sum[i] += v[i];
        if (!e.out)
            return;
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            v[i] = z[i];
    }
    recd_store8(reinterpret_cast<T *>(reinterpret_cast<char *>(e.out) + row * e.out_stride) + col, count, v);
}

__device__ inline void load_bias(const float *bias, int col, int count, float *b)
{
#pragma unroll
    for (int i = 0; i < 8; i++)
        b[i] = 0.0f;
    if (bias)  // (of any alignment of its elements)
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < count)
                b[i] = bias[col + i];
}

// Tiles of one operand from memory through registers into LDS.  COLS: rows of a tile are k, of SIDE columns; else rows are
// the SIDE rows, of BK elements along k, and row f of 32 stands where it is row f of the product (recd_tile_row).  Rows and
// columns behind the operand's end are read from the last one's place: what comes of them is not stored.  Places
// behind k's end are zero.
template <typename T, bool COLS, int SIDE, int BK, int THREADS> struct Loader {
    using Tile = typename std::conditional<COLS, RecdTile<T, BK, SIDE>, RecdTile<T, SIDE, BK>>::type;
    using Piece = typename Tile::Piece;
    static constexpr int E = Tile::E, PR = (COLS ? SIDE : BK) / E, PT = Tile::PIECES / THREADS;
    static_assert(Tile::PIECES % THREADS == 0, "whole pieces a thread");
    Piece held[PT];
    uint32_t off[PT];
    const char *base;

    // `first`: the first row's (COLS: column's) element at the first k
    __device__ inline void begin(int tid, const void *first, uint32_t stride, int left)
    {
        base = reinterpret_cast<const char *>(first);
#pragma unroll
        for (int i = 0; i < PT; i++) {
            const int r = (tid + i * THREADS) / PR, c = (tid + i * THREADS) % PR;
            if constexpr (COLS)
                off[i] = (uint32_t)r * stride + 16u * (uint32_t)(c * E < left ? c : left / E - 1);
            else
                off[i] = (uint32_t)(r < left ? r : left - 1) * stride + 16u * (uint32_t)c;
        }
    }
    // `k_left` > 0: what is left of k from this tile on
    __device__ inline void load(int tid, uint32_t stride, int64_t k_left)
    {
        if (k_left >= BK) {
#pragma unroll
            for (int i = 0; i < PT; i++)
                held[i] = *reinterpret_cast<const Piece *>(base + off[i]);
        } else {
#pragma unroll
            for (int i = 0; i < PT; i++) {
                const int r = (tid + i * THREADS) / PR, c = (tid + i * THREADS) % PR;
                const bool in = COLS ? r < k_left : c * E < k_left;
                const uint32_t back = COLS ? (uint32_t)r * stride : 16u * (uint32_t)c;
                held[i] = *reinterpret_cast<const Piece *>(base + (in ? off[i] : off[i] - back));
                if (!in)
                    held[i] = Piece{};
            }
        }
        base += COLS ? (int64_t)BK * stride : (int64_t)BK * sizeof(T);
    }
    __device__ inline void store(int tid, Tile &t)
    {
#pragma unroll
        for (int i = 0; i < PT; i++) {
            const int r = (tid + i * THREADS) / PR, c = (tid + i * THREADS) % PR;
            t.put_at(COLS ? r : (r & ~31) | recd_tile_row(r & 31), c * E, held[i]);
        }
    }
};

template <typename Tile, bool COLS> __device__ inline auto fragment(const Tile &t, int side, int k, int lane)
{
    if constexpr (COLS)
        return t.columns(k, side, lane);
    else
        return t.rows(side, k, lane);
}

template <typename T, bool COLS, int WI, int WJ, int TI, int TJ, int KIND>
__global__ __launch_bounds__(64 * WI * WJ) void k_product(ProductArgs a)
{
    constexpr int THREADS = 64 * WI * WJ, BI = 32 * WI * TI, BJ = 32 * WJ * TJ, BK = 128 / sizeof(T);
    using Mma = RecdMma<T>;
    using LoadP = Loader<T, COLS, BI, BK, THREADS>;
    using LoadQ = Loader<T, COLS, BJ, BK, THREADS>;
    constexpr int LDW = 32 * TJ + 4;
    __shared__ union {
        struct {
            typename LoadP::Tile p[2];
            typename LoadQ::Tile q[2];
        } t;
        float out[WI * WJ][32 * LDW];
        float cols[WI][BJ];
    } lds;
    // neighbouring tiles on one die, whose L2 then serves what they share: eight tiles of rows by all of the columns, columns slowest
    const int64_t tiles = (int64_t)a.tiles_i * a.tiles_j, total = tiles * a.splits, each = (total + 7) / 8;
    const int64_t at = (int64_t)(blockIdx.x & 7) * each + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= each || at >= total)
        return;
    const int split = (int)(at / tiles), in_split = (int)(at - split * tiles), band = in_split / (8 * a.tiles_j);
    const int in_band = in_split - band * 8 * a.tiles_j, high = a.tiles_i - 8 * band < 8 ? a.tiles_i - 8 * band : 8;
    const int ti = 8 * band + in_band % high, tj = in_band / high;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / WJ, wj = wave % WJ;
    const int64_t i0 = (int64_t)ti * BI, k0 = split * a.k_each, k1 = k0 + a.k_each < a.K ? k0 + a.k_each : a.K;
    const int j0 = tj * BJ;

    recd_f32x16 acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; i++)
#pragma unroll
        for (int j = 0; j < TJ; j++)
            acc[i][j] = recd_f32x16{};
    if (k0 < k1) {
        LoadP lp;
        LoadQ lq;
        const uint32_t ps = (uint32_t)a.p_stride, qs = (uint32_t)a.q_stride;
        const char *p = (const char *)a.p + (COLS ? k0 * a.p_stride + i0 * (int64_t)sizeof(T) : i0 * a.p_stride + k0 * (int64_t)sizeof(T));
        const char *q = (const char *)a.q + (COLS ? k0 * a.q_stride + j0 * (int64_t)sizeof(T) : j0 * a.q_stride + k0 * (int64_t)sizeof(T));
        lp.begin(tid, p, ps, a.n_i - i0 < BI ? (int)(a.n_i - i0) : BI);
        lq.begin(tid, q, qs, a.n_j - j0 < BJ ? a.n_j - j0 : BJ);
        const int64_t steps = (k1 - k0 + BK - 1) / BK;
        lp.load(tid, ps, k1 - k0);
        lq.load(tid, qs, k1 - k0);
        lp.store(tid, lds.t.p[0]);
        lq.store(tid, lds.t.q[0]);
        __syncthreads();
        for (int64_t s = 0; s < steps; s++) {
            const int buf = (int)(s & 1);
            if (s + 1 < steps) {
                lp.load(tid, ps, k1 - k0 - (s + 1) * BK);
                lq.load(tid, qs, k1 - k0 - (s + 1) * BK);
            }
#pragma unroll
            for (int k = 0; k < BK; k += 16) {
                typename Mma::Frag pf[TI], qf[TJ];
#pragma unroll
                for (int i = 0; i < TI; i++)
                    pf[i] = fragment<typename LoadP::Tile, COLS>(lds.t.p[buf], 32 * (wi * TI + i), k, lane);
#pragma unroll
                for (int j = 0; j < TJ; j++)
                    qf[j] = fragment<typename LoadQ::Tile, COLS>(lds.t.q[buf], 32 * (wj * TJ + j), k, lane);
#pragma unroll
                for (int i = 0; i < TI; i++)
#pragma unroll
                    for (int j = 0; j < TJ; j++)
                        acc[i][j] = Mma::mul(qf[j], pf[i], acc[i][j]);
            }
            if (s + 1 < steps) {
                lp.store(tid, lds.t.p[1 - buf]);
                lq.store(tid, lds.t.q[1 - buf]);
            }
            __syncthreads();
        }
    }

    // LPR lanes a row of the wave's columns
    constexpr int LPR = 4 * TJ, RP = 64 / LPR;
    float *mine = lds.out[wave];
    const int piece = lane % LPR, col = j0 + 32 * TJ * wj + 8 * piece;
    const int count = a.n_j - col >= 8 ? 8 : a.n_j - col;
    const bool in = count > 0;
    float b[8], col_sum[8];
    load_bias(KIND != PLAIN && in && !a.part ? a.e.bias : nullptr, col, count, b);
#pragma unroll
    for (int i = 0; i < 8; i++)
        col_sum[i] = 0.0f;
    const uint64_t call = KIND != PLAIN && !a.part ? recd_mask_call(a.e.mask) : 0;
#pragma unroll
    for (int i = 0; i < TI; i++) {
        recd_wave_sync();
#pragma unroll
        for (int j = 0; j < TJ; j++)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<recd_f32x4 *>(mine + (lane & 31) * LDW + 32 * j + recd_sums_row(r, lane)) =
                    recd_f32x4{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
        recd_wave_sync();
#pragma unroll
        for (int pass = 0; pass < 32 / RP; pass++) {
            const int r = pass * RP + lane / LPR;
            const int64_t row = i0 + 32 * (wi * TI + i) + r;
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; e += 4)
                *reinterpret_cast<recd_f32x4 *>(z + e) = *reinterpret_cast<const recd_f32x4 *>(mine + r * LDW + 8 * piece + e);
            if (!in || row >= a.n_i)
                continue;
            if (a.part)
                recd_store8(a.part + ((int64_t)split * a.n_i + row) * a.n_j + col, count, z);
            else
                finish<T, KIND>(a.e, call, row, col, count, a.n_j, b, z, col_sum);
        }
    }
    if constexpr (KIND == GRAD) {
        if (!a.e.col_part || a.part)
            return;
#pragma unroll
        for (int e = 0; e < 8; e++)
#pragma unroll
            for (int o = LPR; o < 64; o <<= 1)
                col_sum[e] += __shfl_xor(col_sum[e], o);
        __syncthreads();
        if (lane < LPR)
#pragma unroll
            for (int e = 0; e < 8; e++)
                lds.cols[wi][32 * TJ * wj + 8 * piece + e] = col_sum[e];
        __syncthreads();
        for (int c = tid; c < BJ; c += THREADS)
            if (j0 + c < a.n_j) {
                float s = 0.0f;
                for (int w = 0; w < WI; w++)
                    s += lds.cols[w][c];
                a.e.col_part[(int64_t)ti * a.n_j + j0 + c] = s;
            }
    }
}

// The same from sums that are there: the splits' in `parts` (added up in their order), or z itself, or none.
struct RowsArgs {
    int64_t n_i;
    int n_j, per_row;      // pieces of eight
    int splits;
    const float *parts;    // [splits][n_i][n_j], or null
    const float *z;        // GRAD: sums that the forward pass kept (with the bias), or null
    int64_t rows_each;     // of a block
    Epilogue e;
};

template <typename T, int KIND> __global__ __launch_bounds__(kBlock) void k_rows(RowsArgs a, int clog)
{
    __shared__ float cols[kBlock][9];
    const int c = threadIdx.x & ((1 << clog) - 1), piece = (blockIdx.x << clog) + c, col = 8 * piece;
    const int count = a.n_j - col >= 8 ? 8 : a.n_j - col;
    const int64_t first = (int64_t)blockIdx.y * a.rows_each, last = first + a.rows_each < a.n_i ? first + a.rows_each : a.n_i;
    float b[8], col_sum[8];
    load_bias(KIND != PLAIN && piece < a.per_row && !a.z ? a.e.bias : nullptr, col, count, b);
#pragma unroll
    for (int i = 0; i < 8; i++)
        col_sum[i] = 0.0f;
    const uint64_t call = KIND != PLAIN ? recd_mask_call(a.e.mask) : 0;
    if (piece < a.per_row)
        for (int64_t row = first + (threadIdx.x >> clog); row < last; row += kBlock >> clog) {
            float z[8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                z[i] = 0.0f;
            if (a.parts)
                for (int s = 0; s < a.splits; s++) {
                    float v[8];
                    recd_load8(a.parts + ((int64_t)s * a.n_i + row) * a.n_j + col, count, v);
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        z[i] += v[i];
                }
            else if (a.z)
                recd_load8(a.z + row * a.n_j + col, count, z);
            finish<T, KIND>(a.e, call, row, col, count, a.n_j, b, z, col_sum);
        }
    if constexpr (KIND == GRAD) {
        if (!a.e.col_part)
            return;
#pragma unroll
        for (int e = 0; e < 8; e++)
            cols[threadIdx.x][e] = col_sum[e];
        __syncthreads();
        // thread t: element t & 7 of the block's piece t >> 3
        for (int t = threadIdx.x; t < 8 << clog; t += kBlock) {
            const int at = (blockIdx.x << clog) * 8 + t;
            if (at >= a.n_j)
                continue;
            float s = 0.0f;
            for (int r = 0; r < kBlock >> clog; r++)
                s += cols[(r << clog) + (t >> 3)][t & 7];
            a.e.col_part[(int64_t)blockIdx.y * a.n_j + at] = s;
        }
    }
}

// Adds up the blocks' column sums in their order: 32 columns by 32 threads, blocks in steps of 32, then the threads' sums.
__global__ __launch_bounds__(1024) void k_join_columns(int64_t blocks, int n_j, const float *__restrict__ part, float *out)
{
    __shared__ float rows[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    float s = 0.0f;
    if (col < n_j)
#pragma unroll 8
        for (int64_t i = r; i < blocks; i += 32)
            s += part[i * n_j + col];
    rows[r][c] = s;
    __syncthreads();
    if (r || col >= n_j)
        return;
    s = 0.0f;
    for (int i = 0; i < 32; i++)
        s += rows[i][c];
    out[col] = s;
}

// Few rows: 16 features a block, whose waves take equal parts of the contraction, straight from memory to the matrix cores; their sums
// are added up in LDS in the waves' order.
constexpr int kFewWaves = 8;

template <typename T> struct Mma16;
template <> struct Mma16<_Float16> {
    using Frag = recd_f16x8;
    static __device__ inline recd_f32x4 mul(Frag a, Frag b, recd_f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma16<__bf16> {
    using Frag = recd_bf16x8;
    static __device__ inline recd_f32x4 mul(Frag a, Frag b, recd_f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma16<float> {
    using Frag = recd_f32x8;
    static __device__ inline recd_f32x4 mul(Frag a, Frag b, recd_f32x4 c)
    {
#pragma unroll
        for (int e = 0; e < 8; e++)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// Elements k .. k + 8 of a row, zero from K on.
template <typename T> __device__ inline typename Mma16<T>::Frag few_frag(const char *row, int k, int K)
{
    constexpr int E = 16 / sizeof(T);
    union {
        typename RecdPiece<T>::type piece[8 / E];
        typename Mma16<T>::Frag f;
    } u;
#pragma unroll
    for (int i = 0; i < 8 / E; i++) {
        u.piece[i] = typename RecdPiece<T>::type{};
        if (k + i * E < K)
            u.piece[i] = *reinterpret_cast<const typename RecdPiece<T>::type *>(row + (k + i * E) * (int)sizeof(T));
    }
    return u.f;
}

template <typename T, int RG> __global__ __launch_bounds__(64 * kFewWaves) void k_few(ProductArgs a)
{
    __shared__ float join[kFewWaves][16 * RG][16 + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = blockIdx.x * 16, n = (int)a.n_i, K = (int)a.K;
    const int j = j0 + (lane & 15) < a.n_j ? j0 + (lane & 15) : a.n_j - 1;
    const char *q = (const char *)a.q + j * a.q_stride;
    const char *p[RG];
#pragma unroll
    for (int g = 0; g < RG; g++) {
        const int i = 16 * g + (lane & 15);
        p[g] = (const char *)a.p + (i < n ? i : n - 1) * a.p_stride;
    }
    recd_f32x4 acc[RG];
#pragma unroll
    for (int g = 0; g < RG; g++)
        acc[g] = recd_f32x4{};
    const int chunks = (K + 31) / 32, each = (chunks + kFewWaves - 1) / kFewWaves;
    const int c1 = (wave + 1) * each < chunks ? (wave + 1) * each : chunks;
#pragma unroll 4
    for (int c = wave * each; c < c1; c++) {
        const int k = 32 * c + 8 * (lane >> 4);
        const auto qf = few_frag<T>(q, k, K);
#pragma unroll
        for (int g = 0; g < RG; g++)
            acc[g] = Mma16<T>::mul(qf, few_frag<T>(p[g], k, K), acc[g]);
    }
#pragma unroll
    for (int g = 0; g < RG; g++)
        *reinterpret_cast<recd_f32x4 *>(&join[wave][16 * g + (lane & 15)][4 * (lane >> 4)]) = acc[g];
    __syncthreads();
    const int row = threadIdx.x >> 1, at = 8 * (threadIdx.x & 1), col = j0 + at;
    if (row >= 16 * RG || row >= n || col >= a.n_j)
        return;
    const int count = a.n_j - col >= 8 ? 8 : a.n_j - col;
    float z[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        z[e] = 0.0f;
        for (int w = 0; w < kFewWaves; w++)
            z[e] += join[w][row][at + e];
    }
    load_bias(a.e.bias, col, count, b);
    finish<T, FORWARD>(a.e, recd_mask_call(a.e.mask), row, col, count, a.n_j, b, z, nullptr);
}

// w [rows, cols] to wt [cols, rows], tiles of 64 x 64.
template <typename T> __global__ __launch_bounds__(kBlock) void k_transpose(int rows, int cols, const T *__restrict__ w, T *__restrict__ wt)
{
    constexpr int E = 16 / sizeof(T), PR = 64 / E;
    using Piece = typename RecdPiece<T>::type;
    __shared__ T tile[64][64 + 2];
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    for (int i = threadIdx.x; i < 64 * PR; i += kBlock) {
        const int r = i / PR, c = i % PR * E;
        if (r0 + r < rows && c0 + c < cols) {
            const Piece v = *reinterpret_cast<const Piece *>(w + (int64_t)(r0 + r) * cols + c0 + c);
            for (int e = 0; e < E; e++)
                tile[r][c + e] = v[e];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * PR; i += kBlock) {
        const int c = i / PR, r = i % PR * E;
        if (c0 + c < cols && r0 + r < rows) {
            Piece v;
            for (int e = 0; e < E; e++)
                v[e] = tile[r + e][c];
            *reinterpret_cast<Piece *>(wt + (int64_t)(c0 + c) * rows + r0 + r) = v;
        }
    }
}

// ---- how a call is cut ---------------------------------------------------------------------------------------------

constexpr int kFewRows = 64;

struct Shape {
    int side;              // rows and columns of a block's tile
    int tiles_i, tiles_j, splits;
    int64_t k_each, turn;  // rows of one launch
};

Shape product_shape(const recd_ctx *ctx, int64_t n_i, int n_j, int64_t K, recd_dtype dt)
{
    const int bk = 128 / (int)elem_size(dt);
    auto tiles = [&](int side) { return ((n_i + side - 1) / side) * ((n_j + side - 1) / side); };
    Shape s;
    s.side = dt != RECD_F32 && tiles(256) >= ctx->num_cu ? 256 : tiles(128) >= ctx->num_cu ? 128 : 64;
    const int64_t cus = 2 * ctx->num_cu, steps = (K + bk - 1) / bk;
    int64_t splits = 1;
    if (tiles(s.side) < ctx->num_cu) {
        splits = cus / tiles(s.side);
        splits = splits < steps / 4 ? splits : steps / 4;
        splits = splits < 1 ? 1 : splits > 256 ? 256 : splits;
    }
    const int64_t each = steps ? (steps + splits - 1) / splits : 1;
    s.k_each = each * bk;
    s.splits = (int)((steps + each - 1) / each);
    if (s.splits < 1)
        s.splits = 1;
    s.tiles_j = (n_j + s.side - 1) / s.side;
    // blocks of one launch: below 2^22
    const int64_t most = ((int64_t)1 << 22) / s.tiles_j * s.side;
    s.turn = s.splits > 1 || n_i <= most ? n_i : most;
    s.tiles_i = (int)((s.turn + s.side - 1) / s.side);
    return s;
}

template <typename T, bool COLS, int KIND> void launch_product(ProductArgs a, const Shape &s, hipStream_t st)
{
    const int64_t n = a.n_i;
    for (int64_t i0 = 0; i0 < n; i0 += s.turn) {
        ProductArgs b = a;
        b.n_i = n - i0 < s.turn ? n - i0 : s.turn;
        b.tiles_i = (int)((b.n_i + s.side - 1) / s.side);
        b.tiles_j = s.tiles_j;
        b.splits = s.splits;
        b.k_each = s.k_each;
        b.p = (const char *)a.p + (COLS ? i0 * (int64_t)sizeof(T) : i0 * a.p_stride);
        if (a.e.other)
            b.e.other = (const char *)a.e.other + i0 * a.e.other_stride;
        if (a.e.out)
            b.e.out = (char *)a.e.out + i0 * a.e.out_stride;
        if (a.e.sums)
            b.e.sums = a.e.sums + i0 * a.n_j;
        if (a.e.col_part)
            b.e.col_part = a.e.col_part + i0 / s.side * a.n_j;
        b.e.row0 = a.e.row0 + i0;
        const dim3 grid((unsigned)(((int64_t)b.tiles_i * b.tiles_j * b.splits + 7) / 8 * 8));
        if (s.side == 256) {
            if constexpr (sizeof(T) == 2)
                hipLaunchKernelGGL((k_product<T, COLS, 2, 4, 4, 2, KIND>), grid, dim3(512), 0, st, b);
        } else if (s.side == 128)
            hipLaunchKernelGGL((k_product<T, COLS, 2, 2, 2, 2, KIND>), grid, dim3(256), 0, st, b);
        else
            hipLaunchKernelGGL((k_product<T, COLS, 2, 2, 1, 1, KIND>), grid, dim3(256), 0, st, b);
    }
}

// Blocks by rows of k_rows, and the log of its pieces a row.
struct RowsShape {
    int clog, groups;
    int64_t blocks, each;
};

RowsShape rows_shape(const recd_ctx *ctx, int64_t n_i, int n_j)
{
    RowsShape s;
    const int pieces = (n_j + 7) / 8;
    s.clog = 0;
    while (s.clog < 5 && 1 << s.clog < pieces)
        s.clog++;
    s.groups = (pieces + (1 << s.clog) - 1) >> s.clog;
    const int at_once = kBlock >> s.clog;
    int64_t blocks = (n_i + at_once - 1) / at_once;
    const int64_t most = ((int64_t)ctx->num_cu * 8 + s.groups - 1) / s.groups;
    blocks = blocks < most ? blocks : most;
    blocks = blocks < 1 ? 1 : blocks;
    s.each = (n_i + blocks - 1) / blocks;
    s.blocks = s.each > 0 ? (n_i + s.each - 1) / s.each : 1;
    if (s.blocks < 1)
        s.blocks = 1;
    return s;
}

template <typename T, int KIND> void launch_rows(const recd_ctx *ctx, RowsArgs a, hipStream_t st)
{
    const RowsShape s = rows_shape(ctx, a.n_i, a.n_j);
    a.per_row = (a.n_j + 7) / 8;
    a.rows_each = s.each;
    hipLaunchKernelGGL((k_rows<T, KIND>), dim3((unsigned)s.groups, (unsigned)s.blocks), dim3(kBlock), 0, st, a, s.clog);
}

// ---- the workspace of a pair of calls --------------------------------------------------------------------------------

struct ForwardPlan {
    bool few;
    Shape shape;
    float *part;

    void make(const recd_ctx *ctx, const recd_dense_layer *a, char *ws, size_t *bytes)
    {
        WsCarver c(ws);
        few = a->n <= kFewRows;
        part = nullptr;
        if (!few) {
            shape = product_shape(ctx, a->n, a->out, a->in, a->dtype);
            if (shape.splits > 1)
                part = c.take<float>((size_t)shape.splits * a->n * a->out);
        }
        *bytes = c.off;
    }
};

struct BackwardPlan {
    bool need_gz, again;   // gz differs from grad_y; z is made again
    Shape z, gx, gw;
    int64_t col_blocks;
    char *gz, *wt;
    float *part, *col_part;  // (one array of parts serves the products in turn)

    void make(const recd_ctx *ctx, const recd_dense_layer *a, bool masked, bool sums, bool grad_x, bool grad_w, bool grad_bias, char *ws,
              size_t *bytes)
    {
        WsCarver c(ws);
        const size_t e = elem_size(a->dtype);
        // (without rows the gradients of w and bias are zero, and nothing is needed for them)
        grad_x = grad_x && a->n > 0;
        need_gz = a->n > 0 && (a->act != RECD_ACT_NONE || masked);
        again = a->n > 0 && a->act != RECD_ACT_NONE && !sums;
        gz = need_gz && (grad_x || grad_w) ? c.take<char>((size_t)a->n * a->out * e) : nullptr;
        wt = grad_x ? c.take<char>((size_t)a->in * a->out * e) : nullptr;
        size_t parts = 0;
        if (again) {
            z = product_shape(ctx, a->n, a->out, a->in, a->dtype);
            if (z.splits > 1)
                parts = larger(parts, (size_t)z.splits * a->n * a->out);
        }
        if (grad_x) {
            gx = product_shape(ctx, a->n, a->in, a->out, a->dtype);
            if (gx.splits > 1)
                parts = larger(parts, (size_t)gx.splits * a->n * a->in);
        }
        if (grad_w) {
            gw = product_shape(ctx, a->out, a->in, a->n, a->dtype);
            if (gw.splits > 1)
                parts = larger(parts, (size_t)gw.splits * a->out * a->in);
        }
        part = parts ? c.take<float>(parts) : nullptr;
        col_blocks = a->n == 0 ? 0 : again && z.splits == 1 ? (a->n + z.side - 1) / z.side : rows_shape(ctx, a->n, a->out).blocks;
        col_part = grad_bias && a->n > 0 ? c.take<float>((size_t)col_blocks * a->out) : nullptr;
        *bytes = c.off;
    }
};

recd_status check_dense(recd_ctx *ctx, const recd_dense_layer *a, RecdMask *mask)
{
    if (!ctx)
        return RECD_EINVAL;
    if (!a)
        return recd_fail(ctx, RECD_EINVAL, "no layer");
    if (a->n < 0 || a->n > ((int64_t)1 << 31) - 1)
        return recd_fail(ctx, RECD_EINVAL, "n=%lld outside [0, 2^31)", (long long)a->n);
    if ((int)a->dtype < 0 || (int)a->dtype > 2)
        return recd_fail(ctx, RECD_EINVAL, "unknown dtype");
    if ((int)a->act < 0 || (int)a->act > RECD_ACT_SILU)
        return recd_fail(ctx, RECD_EINVAL, "unknown activation");
    const int per = 16 / (int)elem_size(a->dtype);
    if (a->in <= 0 || a->out <= 0 || a->in % per || a->out % per || a->in > RECD_MAX_WIDTH || a->out > RECD_MAX_WIDTH)
        return recd_fail(ctx, RECD_EINVAL, "in=%d, out=%d: row bytes must be a multiple of 16, and widths at most %d", a->in, a->out,
                         RECD_MAX_WIDTH);
    return recd_make_mask(ctx, a->dropout, mask);
}

// A row's stride in elements, and where the rows begin.
recd_status check_rows(recd_ctx *ctx, const char *what, const void *p, int64_t stride, int width, recd_dtype dt)
{
    const int64_t e = (int64_t)elem_size(dt);
    if (!p)
        return recd_fail(ctx, RECD_EINVAL, "%s: null pointer argument", what);
    if ((uintptr_t)p % 16 || stride * e % 16 || stride < width || stride * e >= (int64_t)1 << 24)
        return recd_fail(ctx, RECD_EINVAL, "%s: rows of %d must be aligned to 16 bytes, not overlap and lie less than 16 MiB apart", what,
                         width);
    return RECD_OK;
}

} // namespace

extern "C" {

recd_status recd_dense_workspace_bytes(int device, const recd_dense_layer *sizes, size_t *out_bytes)
{
    recd_ctx c;
    RecdMask mask;
    if (!out_bytes)
        return RECD_EINVAL;
    RECD_TRY(check_dense(&c, sizes, &mask));
    RECD_TRY(recd_sizing_context(&c, device));
    *out_bytes = 0;
    if (sizes->n == 0)
        return RECD_OK;
    size_t forward, kept, again;
    ForwardPlan().make(&c, sizes, nullptr, &forward);
    BackwardPlan().make(&c, sizes, mask.cut != 0, true, true, true, true, nullptr, &kept);
    BackwardPlan().make(&c, sizes, mask.cut != 0, false, true, true, true, nullptr, &again);
    *out_bytes = larger(forward, larger(kept, again));
    return RECD_OK;
}

recd_status recd_dense(recd_ctx *ctx, const recd_dense_layer *a, const void *x, const void *w, const float *bias, const void *residual,
                       float *sums, void *y)
{
    RecdMask mask;
    RECD_TRY(check_dense(ctx, a, &mask));
    if (a->n == 0)
        return RECD_OK;
    const int64_t e = (int64_t)elem_size(a->dtype);
    RECD_TRY(check_rows(ctx, "x", x, a->x_stride, a->in, a->dtype));
    RECD_TRY(check_rows(ctx, "w", w, a->in, a->in, a->dtype));
    RECD_TRY(check_rows(ctx, "y", y, a->y_stride, a->out, a->dtype));
    if (residual)
        RECD_TRY(check_rows(ctx, "residual", residual, a->residual_stride, a->out, a->dtype));
    if ((uintptr_t)sums % 16 || (uintptr_t)bias % 4)
        return recd_fail(ctx, RECD_EINVAL, "sums must be aligned to 16 bytes, bias to 4");
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    ForwardPlan plan;
    size_t bytes;
    plan.make(ctx, a, nullptr, &bytes);
    if (bytes) {
        ctx->plan.valid = false;  // the parts overwrite the workspace a backward plan would live in
        RECD_TRY(recd_reserve(ctx, bytes));
        plan.make(ctx, a, ctx->ws, &bytes);
    }
    ProductArgs p{};
    p.n_i = a->n;
    p.n_j = a->out;
    p.K = a->in;
    p.p = x;
    p.q = w;
    p.p_stride = a->x_stride * e;
    p.q_stride = a->in * e;
    p.part = plan.part;
    p.e = Epilogue{(int)a->act, mask, 0, bias, residual, a->residual_stride * e, y, a->y_stride * e, sums, nullptr};
    recd_with_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        if (plan.few) {
            const dim3 grid((unsigned)((a->out + 15) / 16)), block(64 * kFewWaves);
            if (a->n <= 16)
                hipLaunchKernelGGL((k_few<T, 1>), grid, block, 0, ctx->stream, p);
            else if (a->n <= 32)
                hipLaunchKernelGGL((k_few<T, 2>), grid, block, 0, ctx->stream, p);
            else
                hipLaunchKernelGGL((k_few<T, 4>), grid, block, 0, ctx->stream, p);
            return;
        }
        launch_product<T, false, FORWARD>(p, plan.shape, ctx->stream);
        if (plan.part) {
            RowsArgs r{a->n, a->out, 0, plan.shape.splits, plan.part, nullptr, 0, p.e};
            launch_rows<T, FORWARD>(ctx, r, ctx->stream);
        }
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

recd_status recd_dense_backward(recd_ctx *ctx, const recd_dense_layer *a, const void *x, const void *w, const float *bias,
                                const float *sums, const void *grad_y, int64_t grad_y_stride, void *grad_x, int64_t grad_x_stride,
                                void *grad_w, float *grad_bias)
{
    RecdMask mask;
    RECD_TRY(check_dense(ctx, a, &mask));
    const int64_t e = (int64_t)elem_size(a->dtype);
    const int in = a->in, out = a->out;
    if (a->n > 0) {
        const bool again = a->act != RECD_ACT_NONE && !sums;
        RECD_TRY(check_rows(ctx, "grad_y", grad_y, grad_y_stride, out, a->dtype));
        if (again || grad_w)
            RECD_TRY(check_rows(ctx, "x", x, a->x_stride, in, a->dtype));
        if (again || grad_x)
            RECD_TRY(check_rows(ctx, "w", w, in, in, a->dtype));
        if (grad_x)
            RECD_TRY(check_rows(ctx, "grad_x", grad_x, grad_x_stride, in, a->dtype));
    }
    if ((uintptr_t)sums % 16 || (uintptr_t)bias % 4 || (uintptr_t)grad_w % 16 || (uintptr_t)grad_bias % 4)
        return recd_fail(ctx, RECD_EINVAL, "sums and grad_w must be aligned to 16 bytes, bias and grad_bias to 4");
    if ((a->n == 0 || !grad_x) && !grad_w && !grad_bias)
        return RECD_OK;
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    BackwardPlan plan;
    size_t bytes;
    plan.make(ctx, a, mask.cut != 0, sums != nullptr, grad_x != nullptr, grad_w != nullptr, grad_bias != nullptr, nullptr, &bytes);
    if (bytes) {
        ctx->plan.valid = false;
        RECD_TRY(recd_reserve(ctx, bytes));
        plan.make(ctx, a, mask.cut != 0, sums != nullptr, grad_x != nullptr, grad_w != nullptr, grad_bias != nullptr, ctx->ws, &bytes);
    }
    recd_with_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        hipStream_t st = ctx->stream;
        // gz, and its column sums
        const void *gz = plan.gz ? plan.gz : grad_y;
        const int64_t gz_stride = plan.gz ? out * e : grad_y_stride * e;
        Epilogue ep{(int)a->act, mask, 0, bias, grad_y, grad_y_stride * e, plan.gz, out * e, nullptr, plan.col_part};
        if (a->n > 0 && (plan.gz || plan.col_part)) {
            if (plan.again) {
                ProductArgs p{};
                p.n_i = a->n;
                p.n_j = out;
                p.K = in;
                p.p = x;
                p.q = w;
                p.p_stride = a->x_stride * e;
                p.q_stride = in * e;
                p.part = plan.z.splits > 1 ? plan.part : nullptr;
                p.e = ep;
                launch_product<T, false, GRAD>(p, plan.z, st);
            }
            if (!plan.again || plan.z.splits > 1) {
                RowsArgs r{a->n, out, 0, plan.again ? plan.z.splits : 1, plan.again ? plan.part : nullptr, plan.again ? nullptr : sums, 0, ep};
                launch_rows<T, GRAD>(ctx, r, st);
            }
        }
        if (grad_bias)
            hipLaunchKernelGGL(k_join_columns, dim3((unsigned)((out + 31) / 32)), dim3(1024), 0, st, plan.col_blocks, out,
                               plan.col_part, grad_bias);
        if (a->n > 0 && grad_x) {
            hipLaunchKernelGGL((k_transpose<T>), dim3((unsigned)((in + 63) / 64), (unsigned)((out + 63) / 64)), dim3(kBlock), 0, st, out, in,
                               (const T *)w, (T *)plan.wt);
            ProductArgs p{};
            p.n_i = a->n;
            p.n_j = in;
            p.K = out;
            p.p = gz;
            p.q = plan.wt;
            p.p_stride = gz_stride;
            p.q_stride = out * e;
            p.part = plan.gx.splits > 1 ? plan.part : nullptr;
            p.e.out = grad_x;
            p.e.out_stride = grad_x_stride * e;
            launch_product<T, false, PLAIN>(p, plan.gx, st);
            if (p.part) {
                RowsArgs r{a->n, in, 0, plan.gx.splits, p.part, nullptr, 0, p.e};
                launch_rows<T, PLAIN>(ctx, r, st);
            }
        }
        if (grad_w) {
            ProductArgs p{};
            p.n_i = out;
            p.n_j = in;
            p.K = a->n;
            p.p = gz;
            p.q = x;
            p.p_stride = gz_stride;
            p.q_stride = a->x_stride * e;
            p.part = plan.gw.splits > 1 ? plan.part : nullptr;
            p.e.out = grad_w;
            p.e.out_stride = in * e;
            launch_product<T, true, PLAIN>(p, plan.gw, st);
            if (p.part) {
                RowsArgs r{out, in, 0, plan.gw.splits, p.part, nullptr, 0, p.e};
                launch_rows<T, PLAIN>(ctx, r, st);
            }
        }
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

} // extern "C"
