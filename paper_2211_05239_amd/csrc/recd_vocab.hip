// Softmax cross entropy of rows x [n, D] against a whole table [V, D] as the vocabulary, and its gradients.
//
//   z_iv = scale * x_i . W_v,  lse_i = log sum_v exp(z_iv),  loss_i = lse_i - z_i,t(i)
//   p_iv = exp(z_iv - lse_i),  m_i = sum_v p_iv W_v
//   gx_i = scale * g_i * (m_i - W_t(i)),  gW_v = scale * sum_i g_i * (p_iv - [t(i) = v]) * x_i
//
// The logits [n, V] are never stored.  The forward pass streams the table once past rows that stay in registers,
// with a running maximum and sum per row; for training it carries the softmax-weighted mean m_i of the table's rows
// along, as a second product with the scores' exponentials, so that the gradient by x is one subtraction later and
// the backward pass needs one recomputation of the scores instead of two: 8 n V D operations for both passes, where
// 6 are needed at least.  The backward pass turns the sides round: table rows stay in registers, and the rows x
// stream past them.
//
// In 16 bits both passes are bound by the matrix cores and the exponentials beside them.  4096 rows against 1 M x 128 bf16, 4 nVD
// operations a pass: 1.83 ms forward with the mean row (1.15 PFLOP/s) and 2.04 ms for the table's gradient (1.03), at the
// 1.9 GHz that the card's power leaves them, the matrix cores busy 55 % of the cycles; a large product reaches 1.38 PFLOP/s.
// 1500 rows against 100 000 x 64 fp32: 342 and 344 us, 112 TFLOP/s of the 153 of a large product; by count the vector
// instructions take a fifth of the products' cycles there, so what the rest goes to is not shown.
//
// The vocabulary is cut into splits where there are few rows; their (maximum, sum, mean) are joined in the order of the
// splits.  Exponentials are rounded to the tables' type for the second product, as the other operand of the matrix
// cores has it; fp16 ones are scaled by powers of two so that small ones keep their bits.  Sums, maxima and products'
// sums are held in fp32.  Where a row is predicted well its gradients are what is left of 1 - p_t: the table's gradient takes the
// 1 off before rounding, and the mean row's largest weight is exact (kSlack).
#include "recd_internal.h"
#include "recd_mfma.h"

#include <math.h>

namespace {

constexpr int kBlock = 256, kWaves = 4;
// A row's running maximum is moved only where a new one exceeds it by this many powers of two: the exponentials stay
// far inside the range, and the sums are rarely rescaled.  With the mean row in 16 bits that is one power: a logit that has more
// than two thirds of the row's weight then stands at least one above any earlier one, becomes the maximum, and its exponential
// 1 is exact.  The gradient m - W_t of a row that is predicted well is made of the others' weights, and a rounding of
// the target's would be as large as all of them (with a slack of 8, and 1 - p_t = 1 %, the gradient by the row was off by up to 20 %).
template <typename T, bool MEAN> constexpr float kSlack = MEAN && sizeof(T) == 2 ? 1.0f : 8.0f;
// fp16 exponentials are held 2^7 times larger: at most 2^15 with the slack, and exact to 2^-31 of the maximum.
template <typename T> constexpr float kLift = std::is_same<T, _Float16>::value ? 7.0f : 0.0f;

// Tiles of 32 kept rows in a wave, and waves in a block.  Many rows: one tile, since the sums of two take the registers that let
// two waves of a SIMD hide each other's waits, and as many waves as share what they stream; the wide and the fp32 kernels have
// room for four.  Few rows: two tiles a wave, so that a table row that is read feeds both.
template <typename T, int DP> constexpr int kTiles = 1;
template <typename T, int DP> constexpr int kManyWaves = sizeof(T) == 4 || DP > 192 ? 4 : 8;
template <typename T, int DP> constexpr int kFewTiles = sizeof(T) == 4 || DP > 128 ? 1 : 2;

// Rows of a tile that are there, of `left` behind its first.
__device__ inline int rows_left(int64_t left) { return left < 128 ? (int)left : 128; }

// Rows of x that a launch goes through: one holds less than 2^32 threads.
__host__ inline int64_t most_at_once(int64_t n) { return n < (int64_t)1 << 24 ? n : (int64_t)1 << 24; }

struct ForwardArgs {
    int64_t n, V;
    int D;
    float c;            // |scale| * log2(e); the sign goes into the kept side
    bool negative;
    const void *x, *table;
    int row_blocks, splits;
    int64_t tiles_per_split;
    float *part_m, *part_l, *part_o;  // [parts][n] and [parts][n][D]: maximum (in powers of two), sum, weighted sum
};

// Few rows: the block's waves hold the same 32 * N rows and each streams table rows of its own, 32 at a time through LDS
// of its own, so that nobody waits for anybody.  Their sums are joined at the end.  37 rows against 100 000 x 64 fp32 take 15 us
// (25.6 MB, 1.7 TB/s), 32 against 300 000 x 128 bf16 32 (77 MB, 2.4 TB/s): half of what a large copy reaches.  forward_shape gives one
// row block about a hundred splits, so that most compute units have no block at all.
template <typename T, int DP, int N, bool MEAN> __global__ __launch_bounds__(kBlock) void k_vocab_forward_few(ForwardArgs a)
{
    constexpr int KS = DP / 16, DT = DP / 32;
    using Mma = RecdMma<T>;
    using Frag = typename Mma::Frag;
    __shared__ union {
        RecdTile<T, 32, DP> tile[kWaves];
        float join[64 * (2 + (MEAN ? 16 * DT : 0))];
    } lds;
    const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int rb = at % a.row_blocks, split = at / a.row_blocks * 8 + xcd;
    if (split >= a.splits)
        return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = (int64_t)rb * 32 * N;
    const int64_t tiles = (a.V + 127) / 128, t0 = split * a.tiles_per_split;
    const int64_t t1 = t0 + a.tiles_per_split < tiles ? t0 + a.tiles_per_split : tiles;
    RecdTile<T, 32, DP> &tile = lds.tile[wave];

    Frag xf[N][KS];
#pragma unroll
    for (int j = 0; j < N; j++) {
        const int64_t row = row0 + 32 * j + (lane & 31);
#pragma unroll
        for (int k = 0; k < KS; k++) {
            xf[j][k] = recd_row_frag<T>((const T *)a.x + row * a.D, 16 * k, a.D, row < a.n, lane);
            if (a.negative)
                xf[j][k] = recd_negated(xf[j][k]);
        }
    }
    float m[N], l[N];
    recd_f32x16 o[N][MEAN ? DT : 1];
#pragma unroll
    for (int j = 0; j < N; j++) {
        m[j] = -INFINITY;
        l[j] = 0.0f;
#pragma unroll
        for (int d = 0; d < (MEAN ? DT : 1); d++)
            o[j][d] = recd_f32x16{};
    }
    RecdStream<T, 32, DP, 64> stream;
    if (a.D < DP)
        stream.clear_behind(lane, tile, a.D);
    auto load = [&](int64_t t) {
        const int64_t first = t * 128 + 32 * wave;
        if (first < a.V)
            stream.load_rows(lane, (const T *)a.table + first * a.D, rows_left(a.V - first), a.D, a.D * sizeof(T));
    };
    if (t0 < t1)
        load(t0);
    for (int64_t t = t0; t < t1; t++) {
        const int64_t left = a.V - (t * 128 + 32 * wave);
        if (left <= 0)
            break;
        recd_wave_sync();
        stream.store(lane, tile, a.D);
        recd_wave_sync();
        if (t + 1 < t1)
            load(t + 1);
        recd_f32x16 s[N];
#pragma unroll
        for (int j = 0; j < N; j++)
            s[j] = recd_f32x16{};
#pragma unroll
        for (int k = 0; k < KS; k++) {
            const Frag w = tile.rows(0, 16 * k, lane);
#pragma unroll
            for (int j = 0; j < N; j++)
                s[j] = Mma::mul(w, xf[j][k], s[j]);
        }
        if (left < 32) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < N; j++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    s[j][r] = recd_score_row(r, lane) >= (int)left ? -INFINITY : s[j][r];
        }
#pragma unroll
        for (int j = 0; j < N; j++) {
            float top = s[j][0];
#pragma unroll
            for (int r = 1; r < 16; r++)
                top = fmaxf(top, s[j][r]);
            top = fmaxf(top, __shfl_xor(top, 32)) * a.c - kLift<T>;
            if (__any(top > m[j] + kSlack<T, MEAN>)) {
                const float now = fmaxf(m[j], top);
                const float f = now == m[j] ? 1.0f : recd_exp2(m[j] - now);
                m[j] = now;
                l[j] *= f;
                if constexpr (MEAN)
#pragma unroll
                    for (int d = 0; d < DT; d++)
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            o[j][d][r] *= f;
            }
            const float from = m[j] == -INFINITY ? 0.0f : m[j];  // a row of logits that are all -inf
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; r++) {
                s[j][r] = recd_exp2(s[j][r] * a.c - from);
                sum += s[j][r];
            }
            l[j] += sum;
        }
        if constexpr (MEAN) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                Frag p[N];
#pragma unroll
                for (int j = 0; j < N; j++)
                    p[j] = recd_sums_frag<T>(s[j], h);
#pragma unroll
                for (int d = 0; d < DT; d++) {
                    const Frag w = tile.columns(16 * h, 32 * d, lane);
#pragma unroll
                    for (int j = 0; j < N; j++)
                        o[j][d] = Mma::mul(w, p[j], o[j][d]);
                }
            }
        }
    }
    // the waves' sums, in their order, into the first one's
#pragma unroll
    for (int j = 0; j < N; j++) {
        l[j] += __shfl_xor(l[j], 32);
        for (int w = 1; w < kWaves; w++) {
            __syncthreads();
            if (wave == w) {
                lds.join[lane] = m[j];
                lds.join[64 + lane] = l[j];
                if constexpr (MEAN)
#pragma unroll
                    for (int d = 0; d < DT; d++)
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            lds.join[64 * (2 + 16 * d + r) + lane] = o[j][d][r];
            }
            __syncthreads();
            if (wave == 0) {
                const float other = lds.join[lane], top = fmaxf(m[j], other), from = top == -INFINITY ? 0.0f : top;
                const float f = recd_exp2(m[j] - from), g = recd_exp2(other - from);
                m[j] = top;
                l[j] = l[j] * f + lds.join[64 + lane] * g;
                if constexpr (MEAN)
#pragma unroll
                    for (int d = 0; d < DT; d++)
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            o[j][d][r] = o[j][d][r] * f + lds.join[64 * (2 + 16 * d + r) + lane] * g;
            }
        }
    }
    if (wave)
        return;
#pragma unroll
    for (int j = 0; j < N; j++) {
        const int64_t row = row0 + 32 * j + (lane & 31);
        if (row >= a.n)
            continue;
        if (lane < 32) {
            a.part_m[split * a.n + row] = m[j];
            a.part_l[split * a.n + row] = l[j];
        }
        if constexpr (MEAN)
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int col = 32 * d + recd_sums_row(r, lane);
                    if (col < a.D)
                        *reinterpret_cast<recd_f32x4 *>(a.part_o + (split * a.n + row) * a.D + col) =
                            recd_f32x4{o[j][d][r], o[j][d][r + 1], o[j][d][r + 2], o[j][d][r + 3]};
                }
    }
}

// 32 * N rows a wave, other ones in every wave of a block; all of them see every table row of the split.
//
// The loop is pipelined over subtiles of 32 table rows: one turn multiplies the next subtile's scores and the current
// one's sums while the current scores become exponentials, so that matrix cores and vector units have work of one
// basic block to interleave.  The check of the running maximum stands behind it, the only branch.  Three tiles in LDS let
// a wave store the next tile while another one is still at the last but one: one barrier a tile.
template <typename T, int DP, int N, int W, bool MEAN>
__global__ __launch_bounds__(64 * W) void k_vocab_forward(ForwardArgs a)
{
    constexpr int VT = sizeof(T) == 4 && DP > 128 ? 32 : 64;
    constexpr int TURNS = VT / 32;
    constexpr int KS = DP / 16, DT = DP / 32, BUFS = 3;
    using Mma = RecdMma<T>;
    using Frag = typename Mma::Frag;
    __shared__ RecdTile<T, VT, DP> tiles_lds[BUFS];
    // the row blocks of one split side by side on one die, whose L2 then serves the split's rows to all of them
    const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int rb = at % a.row_blocks, split = at / a.row_blocks * 8 + xcd;
    if (split >= a.splits)
        return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = ((int64_t)rb * W + wave) * 32 * N;
    const int64_t tiles = (a.V + VT - 1) / VT, t0 = split * a.tiles_per_split;
    const int64_t t1 = t0 + a.tiles_per_split < tiles ? t0 + a.tiles_per_split : tiles;

    Frag xf[N][KS];
#pragma unroll
    for (int j = 0; j < N; j++) {
        const int64_t row = row0 + 32 * j + (lane & 31);
#pragma unroll
        for (int k = 0; k < KS; k++) {
            xf[j][k] = recd_row_frag<T>((const T *)a.x + row * a.D, 16 * k, a.D, row < a.n, lane);
            if (a.negative)
                xf[j][k] = recd_negated(xf[j][k]);
        }
    }
    float m[N], l[N];
    recd_f32x16 o[N][MEAN ? DT : 1], s[2][N];
#pragma unroll
    for (int j = 0; j < N; j++) {
        m[j] = -INFINITY;
        l[j] = 0.0f;
#pragma unroll
        for (int d = 0; d < (MEAN ? DT : 1); d++)
            o[j][d] = recd_f32x16{};
    }
    auto scores = [&](const RecdTile<T, VT, DP> &tile, int row, recd_f32x16(&out)[N]) {
#pragma unroll
        for (int j = 0; j < N; j++)
            out[j] = recd_f32x16{};
#pragma unroll
        for (int k = 0; k < KS; k++) {
            const Frag w = tile.rows(row, 16 * k, lane);
#pragma unroll
            for (int j = 0; j < N; j++)
                out[j] = Mma::mul(w, xf[j][k], out[j]);
        }
    };
    // rows behind the table's end count as -inf; the maximum moves where new scores are far above it
    auto settle = [&](int64_t v0, recd_f32x16(&x)[N]) {
        if (a.V - v0 < 32) {
            asm volatile("");  // a branch: the last subtile alone pays for the comparisons
            const int left = (int)(a.V - v0);
#pragma unroll
            for (int j = 0; j < N; j++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    x[j][r] = recd_score_row(r, lane) >= left ? -INFINITY : x[j][r];
        }
        float top[N];
        bool above = false;
#pragma unroll
        for (int j = 0; j < N; j++) {
            top[j] = x[j][0];
#pragma unroll
            for (int r = 1; r < 16; r++)
                top[j] = fmaxf(top[j], x[j][r]);
            top[j] = fmaxf(top[j], __shfl_xor(top[j], 32)) * a.c - kLift<T>;
            above |= top[j] > m[j] + kSlack<T, MEAN>;
        }
        if (__any(above))
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float now = fmaxf(m[j], top[j]);
                const float f = now == m[j] ? 1.0f : recd_exp2(m[j] - now);
                m[j] = now;
                l[j] *= f;
                if constexpr (MEAN)
#pragma unroll
                    for (int d = 0; d < DT; d++)
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            o[j][d][r] *= f;
            }
    };
    RecdStream<T, VT, DP, 64 * W> stream;
    if (a.D < DP)
        for (auto &tile : tiles_lds)
            stream.clear_behind(threadIdx.x, tile, a.D);
    auto load = [&](int64_t t) {
        stream.load_rows(threadIdx.x, (const T *)a.table + t * VT * a.D, rows_left(a.V - t * VT), a.D, a.D * sizeof(T));
    };
    if (t0 < t1) {
        load(t0);
        stream.store(threadIdx.x, tiles_lds[0], a.D);
        if (t0 + 1 < t1)
            load(t0 + 1);
        __syncthreads();
        scores(tiles_lds[0], 0, s[0]);
        settle(t0 * VT, s[0]);
    }
    int buf = 0;
    for (int64_t t = t0; t < t1; t++) {
        const int next = buf + 1 == BUFS ? 0 : buf + 1;
        if (t + 1 < t1) {
            stream.store(threadIdx.x, tiles_lds[next], a.D);
            if (t + 2 < t1)
                load(t + 2);
        }
#pragma unroll
        for (int st = 0; st < TURNS; st++) {
            constexpr int kLast = TURNS - 1;
            const int now = TURNS == 1 ? 0 : st & 1, then = TURNS == 1 ? 1 : 1 - now;
            if (st == kLast)
                __syncthreads();
            scores(st == kLast ? tiles_lds[next] : tiles_lds[buf], st == kLast ? 0 : 32 * (st + 1), s[then]);
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float from = m[j] == -INFINITY ? 0.0f : m[j];  // a row of logits that are all -inf
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    s[now][j][r] = recd_exp2(s[now][j][r] * a.c - from);
                    sum += s[now][j][r];
                }
                l[j] += sum;
            }
            if constexpr (MEAN) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    Frag p[N];
#pragma unroll
                    for (int j = 0; j < N; j++)
                        p[j] = recd_sums_frag<T>(s[now][j], h);
#pragma unroll
                    for (int d = 0; d < DT; d++) {
                        const Frag w = tiles_lds[buf].columns(32 * st + 16 * h, 32 * d, lane);
#pragma unroll
                        for (int j = 0; j < N; j++)
                            o[j][d] = Mma::mul(w, p[j], o[j][d]);
                    }
                }
            }
            // behind the last tile these are scores of what an older tile left in LDS, and nobody reads them
            if (st != kLast || t + 1 < t1)
                settle(st == kLast ? (t + 1) * VT : t * VT + 32 * (st + 1), s[then]);
            if constexpr (TURNS == 1)
#pragma unroll
                for (int j = 0; j < N; j++)
                    s[0][j] = s[1][j];
        }
        buf = next;
    }
    const int64_t part = split;
#pragma unroll
    for (int j = 0; j < N; j++) {
        const int64_t row = row0 + 32 * j + (lane & 31);
        const float sum = l[j] + __shfl_xor(l[j], 32);
        if (row >= a.n)
            continue;
        if (lane < 32) {
            a.part_m[part * a.n + row] = m[j];
            a.part_l[part * a.n + row] = sum;
        }
        if constexpr (MEAN)
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int col = 32 * d + recd_sums_row(r, lane);
                    if (col < a.D)
                        *reinterpret_cast<recd_f32x4 *>(a.part_o + (part * a.n + row) * a.D + col) =
                            recd_f32x4{o[j][d][r], o[j][d][r + 1], o[j][d][r + 2], o[j][d][r + 3]};
                }
    }
}

__device__ inline float wave_max(float v)
{
    for (int o = 32; o; o >>= 1)
        v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

__device__ inline float wave_sum(float v)
{
    for (int o = 32; o; o >>= 1)
        v += __shfl_xor(v, o);
    return v;
}

// Joins the parts of a row: a wave per row.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_vocab_join(int64_t n, int64_t V, int D, float scale, int parts,
                                                       const float *__restrict__ part_m, const float *__restrict__ part_l,
                                                       const float *__restrict__ part_o, const T *__restrict__ x,
                                                       const T *__restrict__ table, const int64_t *__restrict__ targets,
                                                       float *loss, float *lse, float *mean_row)
{
    constexpr int E = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (row >= n)
        return;
    // four parts a lane in flight
    float m = -INFINITY, l = 0.0f;
    for (int p0 = lane; p0 < parts; p0 += 256) {
        float pm[4], pl[4], top = m;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const bool there = p0 + 64 * i < parts;
            pm[i] = there ? part_m[(p0 + 64 * i) * n + row] : -INFINITY;
            pl[i] = there ? part_l[(p0 + 64 * i) * n + row] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
            top = fmaxf(top, pm[i]);
        const float from = top == -INFINITY ? 0.0f : top;
        l *= recd_exp2(m - from);
#pragma unroll
        for (int i = 0; i < 4; i++)
            l += recd_exp2(pm[i] - from) * pl[i];
        m = top;
    }
    const float mine = m;
    m = wave_max(m);
    const float from = m == -INFINITY ? 0.0f : m;
    l = wave_sum(l * recd_exp2(mine - from));
    const int64_t t = targets[row];
    float dot = 0.0f;
    if (t >= 0 && t < V)
        for (int v = lane; v < D / E; v += 64) {
            float a[E], b[E];
            recd_load16(x + row * D + v * E, a);
            recd_load16(table + t * D + v * E, b);
            for (int e = 0; e < E; e++)
                dot += a[e] * b[e];
        }
    dot = wave_sum(dot);
    const float total = (m + log2f(l)) * kRecdLn2;
    if (lane == 0) {
        lse[row] = total;
        loss[row] = t >= 0 && t < V ? total - scale * dot : 0.0f;
    }
    if (!mean_row)
        return;
    const float inv = 1.0f / l;
    for (int d = lane; d < D; d += 64) {
        float s = 0.0f;
#pragma unroll 4
        for (int p = 0; p < parts; p++)
            s += recd_exp2(part_m[p * n + row] - from) * part_o[(p * n + row) * D + d];
        mean_row[row * D + d] = s * inv;
    }
}

// The power of two that brings the largest |grad_loss| of the rows with a target into [2^13, 2^14): fp16 products of it with
// probabilities neither overflow nor lose bits that matter beside the largest.
__global__ __launch_bounds__(1024) void k_vocab_lift(int64_t n, int64_t V, const int64_t *__restrict__ targets,
                                                     const float *__restrict__ grad_loss, float *lift)
{
    __shared__ float tops[16];
    float top = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += 1024)
        if ((uint64_t)targets[i] < (uint64_t)V)
            top = fmaxf(top, fabsf(grad_loss[i]));
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0)
        tops[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x)
        return;
    for (int i = 0; i < 16; i++)
        top = fmaxf(top, tops[i]);
    int e = 0;
    frexpf(top, &e);
    e = 14 - (top > 0.0f && top < INFINITY ? e : 14);
    *lift = ldexpf(1.0f, e > 100 ? 100 : e);
}

// What the table's gradient needs of a row (its lse in powers of two, its weight, its target), and the gradient by the row:
// a wave per row, and rows in turns beyond what a launch takes.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_vocab_rows(int64_t n, int64_t V, int D, float scale, const T *__restrict__ table,
                                                       const int64_t *__restrict__ targets, const float *__restrict__ lse,
                                                       const float *__restrict__ mean_row,
                                                       const float *__restrict__ grad_loss, const float *__restrict__ lift,
                                                       float *row_lse, float *row_g, int32_t *row_t, T *grad_x)
{
    constexpr int E = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    for (int64_t row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); row < n; row += (int64_t)gridDim.x * kWaves) {
        const int64_t t = targets[row];
        const bool has = t >= 0 && t < V;
        // (a row whose logits are not all numbers, or one of them infinite, has no gradient that is one)
        const float g = !has ? 0.0f : fabsf(lse[row]) < INFINITY ? grad_loss[row] : NAN;
        if (lane == 0 && row_g) {
            row_lse[row] = has ? lse[row] * kRecdLog2e : INFINITY;
            row_g[row] = lift ? g * *lift : g;
            row_t[row] = has ? (int32_t)t : -1;
        }
        if (!grad_x)
            continue;
        for (int v = lane; v < D / E; v += 64) {
            float a[E], b[E];
            for (int e = 0; e < E; e++)
                a[e] = b[e] = 0.0f;
            if (has) {
                recd_load16(table + t * D + v * E, b);
                for (int e = 0; e < E; e++)
                    a[e] = mean_row[row * D + v * E + e];
            }
            for (int e = 0; e < E; e++)
                a[e] = scale * g * (a[e] - b[e]);
            recd_store16(grad_x + row * D + v * E, a);
        }
    }
}

struct TableGradArgs {
    int64_t n, V;
    int D;
    float c, scale;
    bool negative;
    const void *x, *table;
    const float *row_lse, *row_g, *lift;
    const int32_t *row_t;
    void *grad_table;
    int blocks;        // that share the work (groups of table rows times tiles of rows x) evenly
    float *parts;      // [2 * blocks][rows of a group][D]: sums of groups that several blocks share
};

// 2^x, and 0 for a NaN (the instruction's own clamp): a row without a target, which counts as zeros, has one as its score against a
// table row that holds an infinity.  What a NaN in a score has to do it does by the row's weight.
__device__ inline float probability(float x) { return __builtin_amdgcn_fmed3f(recd_exp2(x), 0.0f, 1.0f); }

// The block that does unit `u` of the work.
__host__ __device__ inline int64_t block_of(int64_t u, int64_t units, int64_t blocks) { return ((u + 1) * blocks - 1) / units; }

// 32 * N table rows a wave; the rows x stream past them, pipelined as in the forward kernel.  A target's weight g (p - 1) enters
// by a product of its own, in the few subtiles that hold a target of the wave's rows: the 1 is taken off before anything is
// rounded, as p and 1 have hardly a bit between them where the model predicts well, and the difference goes in two
// roundings of which the second takes up what the first leaves, as it is most of a row that is a target.
template <typename T, int DP, int N, int W, bool SHARED> __global__ __launch_bounds__(64 * W) void k_vocab_grad_table(TableGradArgs a)
{
    constexpr int XT = sizeof(T) == 4 && DP > 128 ? 32 : 64;
    constexpr int KS = DP / 16, DT = DP / 32, TURNS = XT / 32;
    using Mma = RecdMma<T>;
    using Frag = typename Mma::Frag;
    __shared__ RecdTile<T, XT, DP> tiles_lds[3];
    __shared__ alignas(16) float lse[3][XT], g[3][XT];
    __shared__ int32_t target[3][XT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = (int)((a.n + XT - 1) / XT);
    Frag wf[N][KS];
    recd_f32x16 o[N][DT], s[2][N];
    RecdStream<T, XT, DP, 64 * W> stream;
    if (a.D < DP)
        for (auto &tile : tiles_lds)
            stream.clear_behind(threadIdx.x, tile, a.D);
    float next_lse = 0.0f, next_g = 0.0f;
    int32_t next_t = -1, piece_t[decltype(stream)::PT];
    auto load = [&](int t) {
        const int left = rows_left(a.n - (int64_t)t * XT);
#pragma unroll
        for (int i = 0; i < decltype(stream)::PT; i++) {
            const int r = stream.row(threadIdx.x, i);
            piece_t[i] = (a.row_t + (int64_t)t * XT)[r < left ? r : left - 1];
        }
        stream.load_rows(threadIdx.x, (const T *)a.x + (int64_t)t * XT * a.D, left, a.D, a.D * sizeof(T));
        const int64_t row = (int64_t)t * XT + threadIdx.x;
        const bool there = threadIdx.x < XT && row < a.n;
        next_lse = there ? a.row_lse[row] : INFINITY;  // behind the last row: probability 0
        next_g = there ? a.row_g[row] : 0.0f;
        next_t = there ? a.row_t[row] : -1;
    };
    auto store = [&](int b) {
        // a row without a target may hold anything: it counts as zeros, which no probability turns into a NaN
#pragma unroll
        for (int i = 0; i < decltype(stream)::PT; i++)
            stream.held[i] = piece_t[i] < 0 ? typename decltype(stream)::Piece{} : stream.held[i];
        stream.store(threadIdx.x, tiles_lds[b], a.D);
        if (threadIdx.x < XT) {
            const int i = recd_product_row(threadIdx.x);  // a lane reads those of four neighbouring sums at a time
            lse[b][i] = next_lse;
            g[b][i] = next_g;
            target[b][i] = next_t;
        }
    };
    auto scores = [&](const RecdTile<T, XT, DP> &tile, int row, recd_f32x16(&out)[N]) {
#pragma unroll
        for (int j = 0; j < N; j++)
            out[j] = recd_f32x16{};
#pragma unroll
        for (int k = 0; k < KS; k++) {
            const Frag x = tile.rows(row, 16 * k, lane);
#pragma unroll
            for (int j = 0; j < N; j++)
                out[j] = Mma::mul(x, wf[j][k], out[j]);
        }
    };
    constexpr int R = 32 * N * W;  // table rows of a group
    const float back = a.lift ? a.scale / *a.lift : a.scale;
    const int64_t groups = (a.V + R - 1) / R, units = groups * tiles;
    const int64_t u1 = SHARED ? units * (blockIdx.x + 1) / a.blocks : 0;
    int64_t u = SHARED ? units * blockIdx.x / a.blocks : 0;
    do {
        int64_t group = blockIdx.x;
        int ta = 0, tb = tiles;
        if constexpr (SHARED) {
            group = u / tiles;
            ta = (int)(u - group * tiles);
            if (u1 - u < tiles - ta)
                tb = ta + (int)(u1 - u);
            u += tb - ta;
        }
        const bool whole = !SHARED || (ta == 0 && tb == tiles);
        const int64_t v0 = (group * W + wave) * 32 * N;
#pragma unroll
        for (int j = 0; j < N; j++) {
            const int64_t v = v0 + 32 * j + (lane & 31);
#pragma unroll
            for (int k = 0; k < KS; k++) {
                wf[j][k] = recd_row_frag<T>((const T *)a.table + v * a.D, 16 * k, a.D, v < a.V, lane);
                if (a.negative)
                    wf[j][k] = recd_negated(wf[j][k]);
            }
#pragma unroll
            for (int d = 0; d < DT; d++)
                o[j][d] = recd_f32x16{};
        }
        // the targets among the scores x of subtile st in buffer b: their products, and -inf in the scores' place, whose weight is 0
        auto take_targets = [&](int b, int st, recd_f32x16(&x)[N]) {
            const int32_t mine = target[b][32 * st + (lane & 31)];
            if (!__any(mine >= v0 && mine < v0 + 32 * N))
                return;
#pragma unroll
            for (int j = 0; j < N; j++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    Frag p[2];
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const int r = 8 * h + e, row = 32 * st + recd_sums_row(r, lane);
                        const bool hit = target[b][row] == v0 + 32 * j + (lane & 31);
                        const float w = hit ? (probability(x[j][r] * a.c - lse[b][row]) - 1.0f) * g[b][row] : 0.0f;
                        x[j][r] = hit ? -INFINITY : x[j][r];
                        p[0][e] = (T)w;
                        p[1][e] = (T)(w - (float)p[0][e]);
                    }
#pragma unroll
                    for (int d = 0; d < DT; d++) {
                        const Frag rows = tiles_lds[b].columns(32 * st + 16 * h, 32 * d, lane);
                        o[j][d] = Mma::mul(rows, p[0], o[j][d]);
                        if constexpr (sizeof(T) == 2)
                            o[j][d] = Mma::mul(rows, p[1], o[j][d]);
                    }
                }
        };
        if constexpr (SHARED)
            __syncthreads();  // the last group's readers are through
        if (ta < tb) {
            load(ta);
            store(0);
            if (ta + 1 < tb)
                load(ta + 1);
            __syncthreads();
            scores(tiles_lds[0], 0, s[0]);
        }
        int buf = 0;
        for (int t = ta; t < tb; t++) {
            const int next = buf + 1 == 3 ? 0 : buf + 1;
            if (t + 1 < tb) {
                store(next);
                if (t + 2 < tb)
                    load(t + 2);
            }
#pragma unroll
            for (int st = 0; st < TURNS; st++) {
                constexpr int kLast = TURNS - 1;
                const int now = TURNS == 1 ? 0 : st & 1, then = TURNS == 1 ? 1 : 1 - now;
                take_targets(buf, st, s[now]);
                if (st == kLast)
                    __syncthreads();
                // (behind the last tile: of what an older tile left in LDS, for nobody)
                scores(st == kLast ? tiles_lds[next] : tiles_lds[buf], st == kLast ? 0 : 32 * (st + 1), s[then]);
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int row = 32 * st + recd_sums_row(r, lane);
                    const recd_f32x4 from = *reinterpret_cast<const recd_f32x4 *>(&lse[buf][row]);
                    const recd_f32x4 by = *reinterpret_cast<const recd_f32x4 *>(&g[buf][row]);
#pragma unroll
                    for (int q = 0; q < 4; q++)
#pragma unroll
                        for (int j = 0; j < N; j++)
                            s[now][j][r + q] = probability(s[now][j][r + q] * a.c - from[q]) * by[q];
                }
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    Frag p[N];
#pragma unroll
                    for (int j = 0; j < N; j++)
                        p[j] = recd_sums_frag<T>(s[now][j], h);
#pragma unroll
                    for (int d = 0; d < DT; d++) {
                        const Frag x = tiles_lds[buf].columns(32 * st + 16 * h, 32 * d, lane);
#pragma unroll
                        for (int j = 0; j < N; j++)
                            o[j][d] = Mma::mul(x, p[j], o[j][d]);
                    }
                }
                if constexpr (TURNS == 1)
#pragma unroll
                    for (int j = 0; j < N; j++)
                        s[0][j] = s[1][j];
            }
            buf = next;
        }
#pragma unroll
        for (int j = 0; j < N; j++) {
            const int64_t v = v0 + 32 * j + (lane & 31);
            if (v >= a.V)
                continue;
            float *part = whole ? nullptr : a.parts + ((2 * (int64_t)blockIdx.x + (ta == 0)) * R + (wave * N + j) * 32 + (lane & 31)) * a.D;
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int col = 32 * d + recd_sums_row(r, lane);
                    if (col >= a.D)
                        continue;
                    if (!whole) {
                        *reinterpret_cast<recd_f32x4 *>(part + col) =
                            recd_f32x4{o[j][d][r], o[j][d][r + 1], o[j][d][r + 2], o[j][d][r + 3]};
                        continue;
                    }
                    T out[4];
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        out[q] = (T)(o[j][d][r + q] * back);
                    __builtin_memcpy((T *)a.grad_table + v * a.D + col, out, sizeof out);
                }
        }
    } while (SHARED && u < u1);
}

// Adds up the parts of the groups that several blocks share, in the blocks' order: a block of threads per group.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_vocab_join_table(TableGradArgs a, int R, int64_t each, int64_t units)
{
    const int64_t first = blockIdx.x * each, b0 = block_of(first, units, a.blocks), b1 = block_of(first + each - 1, units, a.blocks);
    if (b0 == b1)
        return;
    const float back = a.lift ? a.scale / *a.lift : a.scale;
    const int64_t v0 = (int64_t)blockIdx.x * R;
    const int rows = a.V - v0 < R ? (int)(a.V - v0) : R, pieces = rows * a.D / 4;
    for (int i = threadIdx.x; i < pieces; i += kBlock) {
        recd_f32x4 s = reinterpret_cast<const recd_f32x4 *>(a.parts + (2 * b0 + 1) * R * a.D)[i];
        for (int64_t b = b0 + 1; b <= b1; b++) {
            const recd_f32x4 x = reinterpret_cast<const recd_f32x4 *>(a.parts + 2 * b * R * a.D)[i];
            for (int e = 0; e < 4; e++)
                s[e] += x[e];
        }
        T out[4];
        for (int e = 0; e < 4; e++)
            out[e] = (T)(s[e] * back);
        __builtin_memcpy((T *)a.grad_table + v0 * a.D + 4 * i, out, sizeof out);
    }
}

// Targets that are no row's sign and lie beyond the table.
__global__ void k_validate_targets(int64_t n, int64_t V, const int64_t *targets, int *err)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x)
        if (targets[i] >= V)
            atomicOr(err, 1);
}

recd_status check_vocab(recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt, float scale)
{
    if (!ctx)
        return RECD_EINVAL;
    if (n < 0 || V < 0 || V > RECD_MAX_VOCAB || n > ((int64_t)1 << 31) - 1)
        return recd_fail(ctx, RECD_EINVAL, "n=%lld outside [0, 2^31) or V=%lld outside [0, %lld]", (long long)n, (long long)V,
                         (long long)RECD_MAX_VOCAB);
    if ((int)dt < 0 || (int)dt > 2)
        return recd_fail(ctx, RECD_EINVAL, "unknown dtype");
    if (!(fabsf(scale) > 0.0f) || !(fabsf(scale) < INFINITY))
        return recd_fail(ctx, RECD_EINVAL, "scale must be finite and not 0");
    if (D <= 0 || D * elem_size(dt) % 16 != 0 || D > RECD_MAX_DENSE_D)
        return recd_fail(ctx, RECD_EINVAL, "D=%d: row bytes must be a multiple of 16, and D at most %d", D, RECD_MAX_DENSE_D);
    return RECD_OK;
}

recd_status validate_targets(recd_ctx *ctx, int64_t n, int64_t V, const int64_t *targets)
{
    ctx->plan.valid = false;
    RECD_TRY(recd_reserve(ctx, RECD_VALIDATE_BYTES));
    int *err = reinterpret_cast<int *>(ctx->ws);
    RECD_HIP(ctx, hipMemsetAsync(err, 0, sizeof(int), ctx->stream));
    hipLaunchKernelGGL(k_validate_targets, dim3(64), dim3(256), 0, ctx->stream, n, V, targets, err);
    RECD_HIP(ctx, hipGetLastError());
    ctx->host_pinned[0] = 0;
    RECD_HIP(ctx, hipMemcpyAsync(ctx->host_pinned, err, sizeof(int), hipMemcpyDeviceToHost, ctx->stream));
    RECD_HIP(ctx, hipStreamSynchronize(ctx->stream));
    if ((int)ctx->host_pinned[0])
        return recd_fail(ctx, RECD_EBOUNDS, "a target is not a row of the table");
    return RECD_OK;
}

// How a forward call is cut: `share` is the kernel of few rows, whose waves stream for themselves and whose rows stay in every
// one of them. In us, it against the other, loss alone and with the mean row: 128 rows bf16 against 300 000 x 128 35, 66 /
// 63, 99; 256 rows 45, 77 / 64, 101; 512 rows 67, 122 / 68, 110; 256 rows fp32 against 100 000 x 64 40, 70 / 51, 91.
struct ForwardShape {
    bool share;
    int row_blocks, splits;
    int64_t tiles_per_split;
};

ForwardShape forward_shape(const recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt, bool mean)
{
    const bool f32 = dt == RECD_F32;
    const int per_few = f32 || D > 128 ? 32 : 64;
    ForwardShape s;
    s.share = n <= 256;
    const int vt = s.share ? 128 : (f32 && D > 128 ? 32 : 64);
    const int64_t rows = s.share ? per_few : (f32 || D > 192 ? 128 : 256), tiles = (V + vt - 1) / vt;
    s.row_blocks = (int)((n + rows - 1) / rows);
    // A die takes every eighth split, all row blocks of it, and holds one or two blocks a CU at a time (the registers of
    // the sums decide): the number of splits whose rounds are fullest, few of them before many whose parts have to
    // be joined; at least two tiles each.  What a split costs is put too high for one row block (100 splits, however large the
    // table), and many rows leave fewer than eight splits and dies without work: bf16 rows of 128 with the mean row from 70 000
    // (7 splits) to 300 000 (one split, one die), fp32 ones from about 50 000.
    const int64_t at_once = (int64_t)ctx->num_cu / 8 * (mean && D > 64 ? 1 : 2);
    int64_t splits = 1;
    double best = 1e30;
    for (int64_t k = 1; k <= 16 * at_once && k * s.row_blocks <= 64 * at_once && (k == 1 || 2 * k <= tiles); k++) {
        const int64_t rounds = ((k + 7) / 8 * s.row_blocks + at_once - 1) / at_once;
        const double cost = (double)rounds / (double)k + 1e-4 * (double)k;
        if (cost < best) {
            best = cost;
            splits = k;
        }
    }
    s.tiles_per_split = (tiles + splits - 1) / splits;
    s.splits = (int)((tiles + s.tiles_per_split - 1) / s.tiles_per_split);
    return s;
}

template <typename T, int DP> void launch_forward(const ForwardArgs &a, bool share, hipStream_t st)
{
    const dim3 grid((unsigned)((a.splits + 7) / 8 * 8 * a.row_blocks));
    const bool mean = a.part_o != nullptr;
    constexpr int N = kTiles<T, DP>, W = kManyWaves<T, DP>;
    if (share && mean)
        hipLaunchKernelGGL((k_vocab_forward_few<T, DP, kFewTiles<T, DP>, true>), grid, dim3(kBlock), 0, st, a);
    else if (share)
        hipLaunchKernelGGL((k_vocab_forward_few<T, DP, kFewTiles<T, DP>, false>), grid, dim3(kBlock), 0, st, a);
    else if (mean)
        hipLaunchKernelGGL((k_vocab_forward<T, DP, N, W, true>), grid, dim3(64 * W), 0, st, a);
    else
        hipLaunchKernelGGL((k_vocab_forward<T, DP, N, W, false>), grid, dim3(64 * W), 0, st, a);
}

// How the table's gradient is cut: blocks that are on the card at a time take equal shares of all (group of table rows,
// tile of rows x) where the last round of whole groups would leave more of the card idle than it costs to write the
// shared groups' parts and add them up (16 bytes an element, at about 4.5 TB/s; the sums run at about 0.9 PFLOP/s, 0.1 in
// fp32), else one block a group.  100 000 x 64 fp32, 1500 rows: 397 us against 447 (782 groups, 512 blocks at a time).
struct TableShape {
    int R;             // table rows of a group
    int64_t each, units;
    int blocks;
    bool shared;
};

template <typename T, int DP> TableShape table_shape(const recd_ctx *ctx, int64_t n, int64_t V, int D)
{
    constexpr int N = kTiles<T, DP>, W = kManyWaves<T, DP>, XT = sizeof(T) == 4 && DP > 128 ? 32 : 64;
    static const int resident = [] {
        int b = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&b, (const void *)k_vocab_grad_table<T, DP, N, W, true>, 64 * W, 0) != hipSuccess) {
            (void)hipGetLastError();
            b = 1;
        }
        return b > 0 ? b : 1;
    }();
    TableShape s;
    s.R = 32 * N * W;
    const int64_t groups = (V + s.R - 1) / s.R, slots = (int64_t)ctx->num_cu * resident;
    s.each = n > 0 ? (n + XT - 1) / XT : 1;
    s.units = groups * s.each;
    const double work = 4.0 * (double)n * (double)V * D / (sizeof(T) == 4 ? 1e14 : 9e14);
    const double idle = (double)((groups + slots - 1) / slots * slots) / (double)groups - 1.0;
    // (a block that may go through several groups is 15 % slower in 16 bits)
    const double gain = (idle - (sizeof(T) == 2 ? 0.15 : 0.0)) * work;
    s.shared = n > 0 && s.units >= slots && gain > (double)(slots * s.R) * D * 16 / 4.5e12 + 5e-6;
    s.blocks = (int)(s.shared ? slots : groups);
    return s;
}

TableShape any_table_shape(const recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt)
{
    TableShape shape{};
    recd_with_type(dt, [&](auto t) { recd_with_width(D, [&](auto w) { shape = table_shape<decltype(t), w.value>(ctx, n, V, D); }); });
    return shape;
}

void carve_parts(WsCarver &c, ForwardArgs &a, bool mean)
{
    a.part_m = c.take<float>((size_t)a.splits * a.n);
    a.part_l = c.take<float>((size_t)a.splits * a.n);
    a.part_o = mean ? c.take<float>((size_t)a.splits * a.n * a.D) : nullptr;
}

struct TableWs {
    float *parts, *row_lse, *row_g, *lift;
    int32_t *row_t;

    void carve(WsCarver &c, const TableShape &shape, int64_t n, int D, recd_dtype dt)
    {
        parts = shape.shared ? c.take<float>((size_t)2 * shape.blocks * shape.R * D) : nullptr;
        row_lse = c.take<float>(n);
        row_g = c.take<float>(n);
        row_t = c.take<int32_t>(n);
        lift = dt == RECD_F16 && n > 0 ? c.take<float>(1) : nullptr;
    }
};

template <typename T, int DP> void launch_grad_table(const TableGradArgs &a, const TableShape &s, hipStream_t st)
{
    constexpr int N = kTiles<T, DP>, W = kManyWaves<T, DP>;
    if (s.shared)
        hipLaunchKernelGGL((k_vocab_grad_table<T, DP, N, W, true>), dim3((unsigned)s.blocks), dim3(64 * W), 0, st, a);
    else
        hipLaunchKernelGGL((k_vocab_grad_table<T, DP, N, W, false>), dim3((unsigned)s.blocks), dim3(64 * W), 0, st, a);
    if (s.shared)
        hipLaunchKernelGGL((k_vocab_join_table<T>), dim3((unsigned)((a.V + s.R - 1) / s.R)), dim3(kBlock), 0, st, a, s.R, s.each,
                           s.units);
}

} // namespace

extern "C" {

recd_status recd_vocab_loss_workspace_bytes(int device, int64_t n, int64_t V, int D, recd_dtype dt, size_t *out_bytes)
{
    recd_ctx c;
    if (!out_bytes)
        return RECD_EINVAL;
    RECD_TRY(check_vocab(&c, n, V, D, dt, 1.0f));
    RECD_TRY(recd_sizing_context(&c, device));
    *out_bytes = 0;
    if (V == 0)
        return RECD_OK;
    size_t most = RECD_VALIDATE_BYTES;
    if (n > 0)
        for (const bool mean : {false, true}) {  // (they are split differently)
            const ForwardShape s = forward_shape(&c, most_at_once(n), V, D, dt, mean);
            ForwardArgs a{};
            a.n = most_at_once(n);
            a.D = D;
            a.splits = s.splits;
            WsCarver parts(nullptr);
            carve_parts(parts, a, mean);
            most = larger(most, parts.off);
        }
    WsCarver table(nullptr);
    TableWs().carve(table, any_table_shape(&c, n, V, D, dt), n, D, dt);
    *out_bytes = larger(most, table.off);
    return RECD_OK;
}

recd_status recd_vocab_loss(recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt, const void *x, const void *table,
                            const int64_t *targets, float scale, float *loss, float *lse, float *mean_row)
{
    RECD_TRY(check_vocab(ctx, n, V, D, dt, scale));
    if (n == 0)
        return RECD_OK;
    if (V == 0)
        return recd_fail(ctx, RECD_EINVAL, "a vocabulary without rows");
    if (!x || !table || !targets || !loss || !lse)
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (((uintptr_t)x | (uintptr_t)table) % 16)
        return recd_fail(ctx, RECD_EINVAL, "x and table must be aligned to 16 bytes");
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    if (ctx->validate)
        RECD_TRY(validate_targets(ctx, n, V, targets));
    ctx->plan.valid = false;  // the parts overwrite the workspace a backward plan would live in
    const int64_t most = most_at_once(n);
    for (int64_t at = 0; at < n; at += most) {
        const int64_t rows = n - at < most ? n - at : most;
        const void *part_x = (const char *)x + at * D * (int64_t)elem_size(dt);
        const ForwardShape s = forward_shape(ctx, rows, V, D, dt, mean_row != nullptr);
        ForwardArgs a{rows, V, D, fabsf(scale) * kRecdLog2e, scale < 0, part_x, table, s.row_blocks, s.splits, s.tiles_per_split};
        WsCarver size(nullptr);
        carve_parts(size, a, mean_row != nullptr);
        RECD_TRY(recd_reserve(ctx, size.off));
        WsCarver c(ctx->ws);
        carve_parts(c, a, mean_row != nullptr);
        recd_with_type(dt, [&](auto t) {
            using T = decltype(t);
            recd_with_width(D, [&](auto w) { launch_forward<T, w.value>(a, s.share, ctx->stream); });
            hipLaunchKernelGGL((k_vocab_join<T>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(kBlock), 0, ctx->stream, rows,
                               V, D, scale, s.splits, a.part_m, a.part_l, a.part_o, (const T *)part_x, (const T *)table,
                               targets + at, loss + at, lse + at, mean_row ? mean_row + at * D : nullptr);
        });
    }
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

recd_status recd_vocab_loss_backward(recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt, const void *x,
                                     const void *table, const int64_t *targets, float scale, const float *lse,
                                     const float *mean_row, const float *grad_loss, void *grad_x, void *grad_table)
{
    RECD_TRY(check_vocab(ctx, n, V, D, dt, scale));
    if (V == 0 && n > 0)
        return recd_fail(ctx, RECD_EINVAL, "a vocabulary without rows");
    if (!grad_x && !grad_table && n > 0)
        return recd_fail(ctx, RECD_EINVAL, "neither grad_x nor grad_table");
    if ((n > 0 && (!x || !targets || !lse || !grad_loss || (grad_x && !mean_row))) || (V > 0 && (n > 0 || grad_table) && !table))
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (((uintptr_t)x | (uintptr_t)table | (uintptr_t)grad_x | (uintptr_t)grad_table) % 16)
        return recd_fail(ctx, RECD_EINVAL, "x, table and their gradients must be aligned to 16 bytes");
    if (V == 0 || (n == 0 && !grad_table))
        return RECD_OK;
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    if (ctx->validate && n > 0)
        RECD_TRY(validate_targets(ctx, n, V, targets));
    TableShape shape{};
    TableWs ws{};
    WsCarver size(nullptr);
    if (grad_table) {
        shape = any_table_shape(ctx, n, V, D, dt);
        ws.carve(size, shape, n, D, dt);
    }
    ctx->plan.valid = false;
    RECD_TRY(recd_reserve(ctx, size.off));
    if (grad_table) {
        WsCarver c(ctx->ws);
        ws.carve(c, shape, n, D, dt);
    }
    float *const row_lse = ws.row_lse, *const row_g = ws.row_g, *const lift = ws.lift;
    int32_t *const row_t = ws.row_t;
    if (lift && n > 0)
        hipLaunchKernelGGL(k_vocab_lift, dim3(1), dim3(1024), 0, ctx->stream, n, V, targets, grad_loss, lift);
    recd_with_type(dt, [&](auto t) {
        using T = decltype(t);
        if (n > 0)
            hipLaunchKernelGGL((k_vocab_rows<T>), dim3((unsigned)((most_at_once(n) + kWaves - 1) / kWaves)), dim3(kBlock), 0, ctx->stream, n,
                               V, D, scale, (const T *)table, targets, lse, mean_row, grad_loss, lift, row_lse, row_g, row_t,
                               (T *)grad_x);
        if (!grad_table)
            return;
        TableGradArgs a{n, V, D, fabsf(scale) * kRecdLog2e, scale, scale < 0, x, table, row_lse, row_g, lift, row_t, grad_table, shape.blocks, ws.parts};
        recd_with_width(D, [&](auto w) { launch_grad_table<T, w.value>(a, shape, ctx->stream); });
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

} // extern "C"
