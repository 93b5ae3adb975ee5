// A dense layer on rows x [n, in] with weights w [out, in], and its gradients.
//
//   z = x w^T + bias,  y = residual + dropout(act(z))
//   gz = dropout'(grad_y) act'(z),  grad_x = gz w,  grad_w = gz^T x,  grad_bias = sum over rows of gz
//
// Every product is C[i, j] = sum over k of P[i, k] Q[j, k].  An operand's rows in memory run along k (both of the layer itself), or along i
// or j (w for grad_x, both for grad_w, which sums over the rows).  Tiles of both go into LDS by loads that write there, a step
// ahead; a wave multiplies TI x TJ tiles of 32 x 32 on the matrix cores, features as the product's rows and rows of x as its columns, so
// that a lane ends up with four neighbouring features of one row.  The sums go through LDS once more: bias, activation, dropout, residual
// and the store work on eight neighbouring features a lane.
//
// What bounds them.  Large products: loads into LDS and the matrix cores beside each other (8192^3 bf16 1.23 PFLOP/s; without the loads
// 2.0, the loads alone as fast as 1.65; the matrix cores are 62 % busy at 1.85 GHz).  16 384 x 8192 -> 1024 with SiLU, both
// directions: 790-835 us for 0.82 TFLOP.  Short contractions: what is done at a tile's end, on the vector units.  300 007 x 128 -> 512 with
// GELU and dropout takes 36 instructions' time an element forward and 44 for gz, GELU more than half of it, with the vector units 73 and 74 %
// busy: 200 us forward, where memory would need 76, 220 for gz; without both 97.  Few rows: w's way from memory, as far as one call's latency lets it (one row 4096 -> 16 384 bf16 5.0 TB/s).
// Small fp32 products: a unit has one or two tiles (5021 x 516 -> 260: 395 tiles of 64, 23 us, of which the matrix cores need 9).
#include "recd_epilogue.h"
#include "recd_mfma.h"

#include <math.h>

namespace {

constexpr int kBlock = 256;

enum { FORWARD = 0, GRAD = 1, PLAIN = 2 };

// What becomes of the sums.  Strides in bytes.
//
// gz is rounded to the layer's type on its way to the gradients' products: the matrix cores take 16-bit operands, and two halves of each
// would be twice the products and twice gz's traffic, for gradients that are rounded to 16 bits themselves (in bf16 they lie 2.3e-3 from the exact
// ones, 1.7e-3 by their own rounding).  grad_bias is summed before the rounding; a layer of fp32 rounds nothing.
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
    const uint32_t *largest;  // fp16, GRAD: k_largest's, or null
    float *unit;              // fp16: what gz is held times; GRAD writes it for what is made of gz (with `largest`), or null
};

// gz of fp16 is held times a power of two of the call, which grad_x and grad_w are divided by: as it is, it would lose digits below 2^-14 and
// vanish below 2^-25, where gradients may well lie that no one has scaled up, and grad_y / (1 - p) could pass 65504.  The power brings the
// largest finite |grad_y| / (1 - p) * 1.13 (no slope is steeper: GELU's is 1.129 at most) to between 2^14 and 2^15, so that whole digits are left down to
// 2^-28 of it, and something down to 2^-39.  It is found by a launch that reads grad_y (300 007 x 128 -> 512 with GELU and dropout, both directions: 581 -> 656 us).  bf16 has the
// range of fp32 and needs none of it.
constexpr int kLargest = 256;  // blocks of k_largest, four a lane here

__device__ inline float gz_unit(const Epilogue &e)
{
    const recd_u32x4 v = *reinterpret_cast<const recd_u32x4 *>(e.largest + 4 * (threadIdx.x & 63));
    uint32_t top = max(max(v[0], v[1]), max(v[2], v[3]));
#pragma unroll
    for (int o = 32; o; o >>= 1)
        top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if (top == 0)
        return 1.0f;
    const float bound = (float)__builtin_bit_cast(_Float16, (unsigned short)top) * e.mask.by * 1.13f;
    return ldexpf(1.0f, 15 - (int)((__builtin_bit_cast(uint32_t, bound) >> 23) - 126u));
}

// What the sums are multiplied by on their way out.  `first`: one block of the call's.
template <typename T, int KIND> __device__ inline float unit_of(const Epilogue &e, bool first)
{
    if constexpr (std::is_same<T, _Float16>::value && KIND == GRAD) {
        if (e.largest) {
            const float unit = gz_unit(e);
            if (first && threadIdx.x == 0)
                *e.unit = unit;
            return unit;
        }
    } else if constexpr (std::is_same<T, _Float16>::value && KIND == PLAIN) {
        if (e.unit)
            return 1.0f / *e.unit;
    }
    return 1.0f;
}

// Block by block, the largest finite |g| of rows [n, 8 * per_row], as the bits of an fp16.
__global__ __launch_bounds__(1024) void k_largest(int64_t n, int per_row, const char *g, int64_t stride, uint32_t *out)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    __shared__ uint32_t tops[16];
    // from the last row to the first, which the next launch then finds in the caches: `at` counts from the end
    const int64_t pieces = n * per_row, threads = (int64_t)kLargest * 1024, drow = threads / per_row;
    const int dcol = (int)(threads - drow * per_row);
    int64_t at = (int64_t)blockIdx.x * 1024 + threadIdx.x, row = at / per_row;
    int col = (int)(at - row * per_row);
    u16x2 top = {0, 0};
    while (at < pieces) {
        recd_u32x4 v[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v[i] = recd_u32x4{};
            if (at + i * threads < pieces)
                v[i] = *reinterpret_cast<const recd_u32x4 *>(g + (n - 1 - row) * stride + 16 * col);
            row += drow;
            col += dcol;
            if (col >= per_row) {
                col -= per_row;
                row++;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const u16x2 b = __builtin_bit_cast(u16x2, v[i][w] & 0x7fff7fffu);
                top = __builtin_elementwise_max(top, u16x2{(unsigned short)(b[0] < 0x7c00 ? b[0] : 0), (unsigned short)(b[1] < 0x7c00 ? b[1] : 0)});
            }
        at += 4 * threads;
    }
    uint32_t all = top[0] > top[1] ? top[0] : top[1];
    for (int o = 32; o; o >>= 1)
        all = max(all, (uint32_t)__shfl_xor((int)all, o));
    if ((threadIdx.x & 63) == 0)
        tops[threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; w++)
            all = max(all, tops[w]);
        out[blockIdx.x] = all;
    }
}

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

// Eight neighbouring elements of a row, as they lie in memory.
template <typename T> struct Eight {
    typename RecdPiece<T>::type piece[sizeof(T) / 2];
    __device__ inline void load(const char *at, int count)
    {
        using Piece = typename RecdPiece<T>::type;
        piece[0] = *reinterpret_cast<const Piece *>(at);
        if constexpr (sizeof(T) == 4)
            piece[1] = count == 8 ? *reinterpret_cast<const Piece *>(at + 16) : Piece{};
    }
    __device__ inline float operator[](int e) const { return (float)piece[e * (int)sizeof(T) / 16][e % (16 / (int)sizeof(T))]; }
};

template <typename T> __device__ inline void store_half(T *to, int half, const float *v)
{
    typedef T T4 __attribute__((ext_vector_type(4)));
    const float *h = half ? v + 4 : v;
    *reinterpret_cast<T4 *>(to + 4 * half) = T4{(T)h[0], (T)h[1], (T)h[2], (T)h[3]};
}

// Eight (`count`) sums of row `row` from column `col` on.  `b`: the columns' bias, `other`: the residual's or grad_y's elements.  `half`: the
// one half of them that is wanted (FORWARD), or -1.
template <typename T, int KIND>
__device__ inline void finish(const Epilogue &e, const RecdBits &bits, int64_t row, int col, int count, int n_j, const float *b, float *z,
                              const Eight<T> &other, float *col_sum, float unit = 1.0f, int half = -1)
{
    float v[8];
    if constexpr (KIND == FORWARD) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            v[i] = z[i] + b[i];
        if (e.sums && half < 0)
            recd_store8(e.sums + row * n_j + col, count, v);
        else if (e.sums)
            store_half(e.sums + row * n_j + col, half, v);
        recd_activate(e.act, v);
        if (e.mask.cut)
            recd_mask_apply(e.mask, bits, v);
        if (e.other)
#pragma unroll
            for (int i = 0; i < 8; i++)
                v[i] += other[i];
    } else if constexpr (KIND == GRAD) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            v[i] = e.mask.cut ? other[i] * e.mask.by : other[i];
        if (e.act != RECD_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                z[i] += b[i];
            recd_activate_back(e.act, z, v);
        }
        if (e.mask.cut)  // (last: the slope of a z that is not finite may be a NaN, and what is dropped is 0 whatever z is)
            recd_mask_drop(e.mask, bits, v);
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
    if constexpr (std::is_same<T, _Float16>::value && KIND != FORWARD)
#pragma unroll
        for (int i = 0; i < 8; i++)
            v[i] *= unit;
    T *to = reinterpret_cast<T *>(reinterpret_cast<char *>(e.out) + row * e.out_stride) + col;
    if (half < 0)
        recd_store8_past(to, count, v);
    else
        store_half(to, half, v);
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

// A quarter of a step of the contraction: 16 bytes of k of a row in each half wave.
template <typename T> struct Quarter {
    using Frag = typename RecdMma<T>::Frag;
    static __device__ inline recd_f32x16 mul(Frag a, Frag b, recd_f32x16 c) { return RecdMma<T>::mul(a, b, c); }
};
template <> struct Quarter<float> {
    using Frag = recd_f32x4;
    static __device__ inline recd_f32x16 mul(Frag a, Frag b, recd_f32x16 c)
    {
#pragma unroll
        for (int e = 0; e < 4; e++)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// Tiles of one operand, two of them in LDS, which the loads write to by themselves.  COLS: a tile's rows are BK values of k, of SIDE
// columns; else they are the SIDE rows, of BK elements along k (128 bytes: shorter ones ask the L2 twice for each line).  Rows and
// columns behind the operand's end are read from the last one's place: what comes of them is not stored.
//
// A load of a wave fills 1024 bytes of LDS in its lanes' order; which 16 bytes of memory a lane brings is free.  So that the
// lanes that read at a time meet in no bank, piece c of row r stands at place c ^ (r >> 1 & 7) of the row (reads of one piece from 16 rows), and
// with COLS 64-byte segment s at place s ^ (r & 3 ^ r >> 2 & 2) (transposing reads take a segment of four rows at a time; 32-bit ones two
// segments of rows 4 apart, with r >> 1); rows of 128 bytes, two segments of which take the banks, at place s ^ (r >> 1 & 1).
template <typename T, bool COLS, int SIDE, int WAVES> struct Operand {
    using Piece = typename RecdPiece<T>::type;
    using Frag = typename Quarter<T>::Frag;
    static constexpr int E = 16 / sizeof(T), BK = 128 / sizeof(T), BYTES = SIDE * 128, ROW = COLS ? SIDE * (int)sizeof(T) : 128;
    static constexpr int PT = BYTES / 1024 / WAVES;  // loads of a wave
    static_assert(BYTES % (1024 * WAVES) == 0, "whole loads a wave");
    uint32_t off[PT];
    const char *base;

    static __device__ inline int turn(int r)
    {
        if constexpr (!COLS)
            return r >> 1 & 7;
        else if constexpr (ROW == 128)
            return (r >> 1 & 1) << 2;
        else
            return ((r & 3) ^ (sizeof(T) == 4 ? r >> 1 & 2 : r >> 2 & 2)) << 2;
    }
    // row and piece of a lane's bytes of the wave's load i
    static __device__ inline void place(int wave, int lane, int i, int &r, int &c)
    {
        const int at = (wave * PT + i) * 1024 + lane * 16;
        r = at / ROW;
        c = (at % ROW / 16) ^ turn(r);
    }
    // `first`: the first row's (COLS: column's) element at the first k; `left` rows (columns) are there
    __device__ inline void begin(int wave, int lane, const char *first, uint32_t stride, int left)
    {
        base = first;
#pragma unroll
        for (int i = 0; i < PT; i++) {
            int r, c;
            place(wave, lane, i, r, c);
            if constexpr (COLS)
                off[i] = (uint32_t)r * stride + 16u * (uint32_t)(c * E < left ? c : left / E - 1);
            else
                off[i] = (uint32_t)(r < left ? r : left - 1) * stride + 16u * (uint32_t)c;
        }
    }
    __device__ inline void step(uint32_t stride) { base += COLS ? (int64_t)BK * stride : 128; }
    // the wave's load i of a tile, all of which is there: waited for by vmcnt
    __device__ inline void send(char *to, int wave, int i) const
    {
        using Global = const __attribute__((address_space(1))) void;
        using Local = __attribute__((address_space(3))) void;
        __builtin_amdgcn_global_load_lds((Global *)(base + off[i]), (Local *)(to + (wave * PT + i) * 1024), 16, 0, 0);
    }
    // the last tile, of which `k_left` > 0 are there and zeros stand behind them: through registers
    __device__ inline void bring(char *to, int wave, int lane, uint32_t stride, int k_left)
    {
#pragma unroll
        for (int i = 0; i < PT; i++) {
            int r, c;
            place(wave, lane, i, r, c);
            const bool in = COLS ? r < k_left : c * E < k_left;
            const uint32_t back = COLS ? (uint32_t)r * stride : 16u * (uint32_t)c;
            Piece v = *reinterpret_cast<const Piece *>(base + (in ? off[i] : off[i] - back));
            if (!in)
                v = Piece{};
            *reinterpret_cast<Piece *>(to + (wave * PT + i) * 1024 + lane * 16) = v;
        }
    }
    // rows (columns) side .. side + 32 as the product has them, a quarter of the tile's k: 16 bytes of it in each half wave
    static __device__ inline Frag fragment(const char *from, int side, int quarter, int lane)
    {
        const int k = quarter * BK / 4 + (lane >> 5) * E;
        if constexpr (!COLS) {
            const int r = side + (lane & 31);
            return *reinterpret_cast<const Piece *>(from + r * ROW + 16 * ((k / E) ^ turn(r)));
        } else if constexpr (sizeof(T) == 4) {
            Frag f;
            const int col = side + (lane & 31);
#pragma unroll
            for (int e = 0; e < E; e++)
                f[e] = *reinterpret_cast<const T *>(from + (k + e) * ROW + 16 * ((col / E) ^ turn(k + e)) + 4 * (col % E));
            return f;
        } else {
            // 16 lanes name four rows of 16 columns, 8 bytes each; each of them receives one column
            using Half4 = __attribute__((address_space(3))) recd_s16x4;
            const int i = lane & 15, col = side + 16 * (lane >> 4 & 1) + 4 * (i & 3);
            union {
                recd_s16x4 four[2];
                Frag f;
            } u;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int r = k + 4 * h + (i >> 2);
                u.four[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half4 *)(from + r * ROW + 16 * ((col / E) ^ turn(r)) + 2 * (col % E)));
            }
            return u.f;
        }
    }
};

// The wave's loads into LDS, but for the last N, have arrived and its LDS reads and writes are done, and that holds for all waves of
// the block.
template <int N = 0> __device__ inline void arrive()
{
    static_assert(N < 16);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_s_waitcnt(N | 7 << 4);  // vmcnt N, lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Two tiles of each operand, then the sums on their way out.
template <int WI, int WJ, int TI, int TJ> union ProductLds {
    struct {
        alignas(16) char p[2][32 * WI * TI * 128];
        alignas(16) char q[2][32 * WJ * TJ * 128];
    } t;
    float out[WI * WJ][32 * (32 * TJ + 4)];
    float cols[WI][32 * WJ * TJ];
};

// Block `block` of a product.
template <typename T, bool PCOLS, bool QCOLS, int WI, int WJ, int TI, int TJ, int KIND>
__device__ inline void product(ProductArgs a, unsigned block, ProductLds<WI, WJ, TI, TJ> &lds)
{
    constexpr int THREADS = 64 * WI * WJ, BI = 32 * WI * TI, BJ = 32 * WJ * TJ;
    using P = Operand<T, PCOLS, BI, WI * WJ>;
    using Q = Operand<T, QCOLS, BJ, WI * WJ>;
    constexpr int BK = P::BK, LDW = 32 * TJ + 4;
    // neighbouring tiles on one die, whose L2 then serves what they share: eight tiles of rows by all of the columns, columns slowest
    const int64_t tiles = (int64_t)a.tiles_i * a.tiles_j, total = tiles * a.splits, each = (total + 7) / 8;
    const int64_t at = (int64_t)(block & 7) * each + (block >> 3);
    if ((int64_t)(block >> 3) >= each || at >= total)
        return;
    const int split = (int)(at / tiles), in_split = (int)(at - split * tiles), band = in_split / (8 * a.tiles_j);
    const int in_band = in_split - band * 8 * a.tiles_j, high = a.tiles_i - 8 * band < 8 ? a.tiles_i - 8 * band : 8;
    const int ti = 8 * band + in_band % high, tj = in_band / high;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / WJ, wj = wave % WJ;
    const int64_t i0 = (int64_t)ti * BI, k0 = split * a.k_each, k1 = k0 + a.k_each < a.K ? k0 + a.k_each : a.K;
    const int j0 = tj * BJ, rows = a.n_i - i0 < BI ? (int)(a.n_i - i0) : BI;

    // LPR lanes a row of the wave's columns, eight columns each, RP rows at a time
    constexpr int LPR = 4 * TJ, RP = 64 / LPR, PASSES = 32 / RP;
    const int piece = lane % LPR, col = j0 + 32 * TJ * wj + 8 * piece;
    const int count = a.n_j - col >= 8 ? 8 : a.n_j - col;
    const bool in = count > 0;
    // the residual's or grad_y's elements of the wave's rows 32 i .. 32 i + 32, on their way before they are needed
    Eight<T> other[PASSES];
    const bool with_other = KIND != PLAIN && in && !a.part && a.e.other;
    auto fetch = [&](int i) {
        if (with_other)
#pragma unroll
            for (int pass = 0; pass < PASSES; pass++) {
                const int r = 32 * (wi * TI + i) + pass * RP + lane / LPR;
                if (r < rows)
                    other[pass].load(reinterpret_cast<const char *>(a.e.other) + i0 * a.e.other_stride + (uint32_t)r * (uint32_t)a.e.other_stride +
                                         (uint32_t)col * (uint32_t)sizeof(T),
                                     count);
            }
    };
    fetch(0);

    recd_f32x16 acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; i++)
#pragma unroll
        for (int j = 0; j < TJ; j++)
            acc[i][j] = recd_f32x16{};
    if (k0 < k1) {
        P lp;
        Q lq;
        const uint32_t ps = (uint32_t)a.p_stride, qs = (uint32_t)a.q_stride;
        lp.begin(wave, lane, (const char *)a.p + (PCOLS ? k0 * a.p_stride + i0 * (int64_t)sizeof(T) : i0 * a.p_stride + k0 * (int64_t)sizeof(T)), ps, rows);
        lq.begin(wave, lane, (const char *)a.q + (QCOLS ? k0 * a.q_stride + j0 * (int64_t)sizeof(T) : j0 * a.q_stride + k0 * (int64_t)sizeof(T)), qs,
                 a.n_j - j0 < BJ ? a.n_j - j0 : BJ);
        const int whole = (int)((k1 - k0) / BK), tail = (int)((k1 - k0) % BK), steps = whole + (tail ? 1 : 0);
        // loads from .. to of the tile that comes next, which goes to place `buf`: first P's, then Q's
        constexpr int LOADS = P::PT + Q::PT;
        auto send = [&](int buf, int from, int to) {
#pragma unroll
            for (int i = from; i < to; i++)
                if (i < P::PT)
                    lp.send(lds.t.p[buf], wave, i);
                else
                    lq.send(lds.t.q[buf], wave, i - P::PT);
        };
        auto sent = [&] {
            lp.step(ps);
            lq.step(qs);
        };
        auto bring = [&](int buf) {
            lp.bring(lds.t.p[buf], wave, lane, ps, tail);
            lq.bring(lds.t.q[buf], wave, lane, qs, tail);
        };
        typename Quarter<T>::Frag pf[2][TI], qf[2][TJ];
        auto read = [&](int s, int quarter) {
#pragma unroll
            for (int i = 0; i < TI; i++)
                pf[quarter & 1][i] = P::fragment(lds.t.p[s & 1], 32 * (wi * TI + i), quarter, lane);
#pragma unroll
            for (int j = 0; j < TJ; j++)
                qf[quarter & 1][j] = Q::fragment(lds.t.q[s & 1], 32 * (wj * TJ + j), quarter, lane);
        };
        // A step: four quarters, whose fragments are read while the matrix cores have the quarter before.  Before the last one the
        // next tile is there and this one has been read, whose place the next but one takes: its loads go out between the
        // products of that quarter, as the matrix cores would wait for a row of them to be taken (8192^3: 1.02 PFLOP/s in a row, 1.24
        // between; spread over two quarters some arrive late, 3 % less in the gradients).
        auto step = [&](int s, auto more) {
#pragma unroll
            for (int quarter = 0; quarter < 4; quarter++) {
                if (quarter < 3)
                    read(s, quarter + 1);
                else {
                    arrive();
                    if (s + 2 == whole && tail)
                        bring(s & 1);
                    read(s + 1, 0);  // (behind the last tile: what an older one left, for nobody)
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < TI; i++)
#pragma unroll
                    for (int j = 0; j < TJ; j++) {
                        constexpr int MANY = TI * TJ;
                        const int m = i * TJ + j;
                        acc[i][j] = Quarter<T>::mul(qf[quarter & 1][j], pf[quarter & 1][i], acc[i][j]);
                        __builtin_amdgcn_sched_barrier(0);
                        if (more.value && quarter == 3) {
                            send(s & 1, m * LOADS / MANY, (m + 1) * LOADS / MANY);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
            }
        };
        if (whole > 0) {
            send(0, 0, LOADS);
            sent();
        } else
            bring(0);
        if (whole > 1) {
            send(1, 0, LOADS);
            sent();
            arrive<LOADS>();
        } else {
            if (whole == 1 && tail)
                bring(1);
            arrive();
        }
        read(0, 0);
        int s = 0;
        for (; s + 2 < whole; s++) {
            step(s, std::true_type{});
            sent();
        }
        for (; s < steps; s++)
            step(s, std::false_type{});
        arrive();
    }

    float *mine = lds.out[wave];
    float b[8], col_sum[8];
    load_bias(KIND != PLAIN && in && !a.part ? a.e.bias : nullptr, col, count, b);
#pragma unroll
    for (int i = 0; i < 8; i++)
        col_sum[i] = 0.0f;
    const bool masked = KIND != PLAIN && !a.part && a.e.mask.cut;
    const float unit = a.part ? 1.0f : unit_of<T, KIND>(a.e, block == 0);
    const RecdMaskPiece mask = masked ? recd_mask_piece(a.e.mask, recd_mask_call(a.e.mask), col >> 3) : RecdMaskPiece{};
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
        Eight<T> now[PASSES];
#pragma unroll
        for (int pass = 0; pass < PASSES; pass++)
            now[pass] = other[pass];
        if (i + 1 < TI)
            fetch(i + 1);
        // all of the masks' bits beside each other: a row's rounds wait for each other
        RecdBits bits[PASSES] = {};
        if (masked)
#pragma unroll
            for (int pass = 0; pass < PASSES; pass++)
                bits[pass] = recd_mask_bits(a.e.mask, mask, (uint32_t)(a.e.row0 + i0) + (uint32_t)(32 * (wi * TI + i) + pass * RP + lane / LPR));
#pragma unroll
        for (int pass = 0; pass < PASSES; pass++) {
            const int in_wave = pass * RP + lane / LPR, r = 32 * (wi * TI + i) + in_wave;
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; e += 4)
                *reinterpret_cast<recd_f32x4 *>(z + e) = *reinterpret_cast<const recd_f32x4 *>(mine + in_wave * LDW + 8 * piece + e);
            if (!in || r >= rows)
                continue;
            if (a.part)
                recd_store8(a.part + ((int64_t)split * a.n_i + i0 + r) * a.n_j + col, count, z);
            else
                finish<T, KIND>(a.e, bits[pass], i0 + r, col, count, a.n_j, b, z, now[pass], col_sum, unit);
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

template <typename T, bool PCOLS, bool QCOLS, int WI, int WJ, int TI, int TJ, int KIND>
__global__ __launch_bounds__(64 * WI * WJ) void k_product(ProductArgs a)
{
    __shared__ ProductLds<WI, WJ, TI, TJ> lds;
    product<T, PCOLS, QCOLS, WI, WJ, TI, TJ, KIND>(a, blockIdx.x, lds);
}

// The gradients of x and w in one launch, where both have the same tile: the blocks of one fill what the other would leave idle at its end.
// The `blocks_w` of w's gradient come first, as they mostly take longer.  Both, us in two launches and in one: 512 x 512 -> 512 bf16 12.0
// and 9.2, 2000 x 128 -> 512 bf16 14.8 and 12.2, 300 x 2048 -> 512 fp32 25.3 and 20.5, 5021 x 516 -> 260 fp32 50.1 and 45.7, 300 007 x 128 ->
// 512 bf16 177 and 166; tiles of 256, one of which fills a unit, stay in two (16 384 x 8192 -> 1024 bf16 with gz and the sums 776 and 800).
template <typename T, int WI, int WJ, int TI, int TJ>
__global__ __launch_bounds__(64 * WI * WJ) void k_gradients(ProductArgs x, ProductArgs w, unsigned blocks_w)
{
    __shared__ ProductLds<WI, WJ, TI, TJ> lds;
    if (blockIdx.x < blocks_w)
        product<T, true, true, WI, WJ, TI, TJ, PLAIN>(w, blockIdx.x, lds);
    else
        product<T, false, true, WI, WJ, TI, TJ, PLAIN>(x, blockIdx.x - blocks_w, lds);
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
    const float unit = unit_of<T, KIND>(a.e, blockIdx.x == 0 && blockIdx.y == 0);
    const RecdMaskPiece mask = KIND != PLAIN && a.e.mask.cut ? recd_mask_piece(a.e.mask, recd_mask_call(a.e.mask), piece) : RecdMaskPiece{};
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
            Eight<T> other{};
            if (KIND != PLAIN && a.e.other)
                other.load(reinterpret_cast<const char *>(a.e.other) + row * a.e.other_stride + (int64_t)col * sizeof(T), count);
            const RecdBits bits = KIND != PLAIN && a.e.mask.cut ? recd_mask_bits(a.e.mask, mask, (uint32_t)(a.e.row0 + row)) : RecdBits{};
            finish<T, KIND>(a.e, bits, row, col, count, a.n_j, b, z, other, col_sum, unit);
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

// A product of SLICES splits or more: 64 pieces of eight sums a block, whose waves add up equal parts of the splits in their order; the
// waves' sums then go through LDS, in order too.  One lane after the other split, as k_rows has it, waits for memory each time and
// leaves most of the card idle where the sums are few (grad_w of 300 007 x 64 -> 64 bf16 81 us, here 23; of 128 -> 512 123 and 110; 27 rows
// 5844 -> 60 fp32 20.5 and 10.5, 100 rows 8192 -> 256 bf16 17.0 and 10.2); four waves 26 and 110 for the first two, sixteen 24 and 112.
constexpr int SLICES = 8;

template <typename T, int KIND> __global__ __launch_bounds__(64 * SLICES) void k_join(RowsArgs a)
{
    __shared__ float sums[SLICES][64][8 + 1];
    const int lane = threadIdx.x & 63, slice = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t at = (int64_t)blockIdx.x * 64 + lane, row = at / a.per_row;
    const int col = 8 * (int)(at - row * a.per_row), count = a.n_j - col >= 8 ? 8 : a.n_j - col;
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; e++)
        z[e] = 0.0f;
    if (row < a.n_i) {
        const int each = (a.splits + SLICES - 1) / SLICES, last = (slice + 1) * each < a.splits ? (slice + 1) * each : a.splits;
#pragma unroll 4
        for (int s = slice * each; s < last; s++) {
            float v[8];
            recd_load8(a.parts + ((int64_t)s * a.n_i + row) * a.n_j + col, count, v);
#pragma unroll
            for (int e = 0; e < 8; e++)
                z[e] += v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        sums[slice][lane][e] = z[e];
    __syncthreads();
    if (slice || row >= a.n_i)
        return;
    const float unit = unit_of<T, KIND>(a.e, false);  // (of gz itself column sums are taken besides: never here)
    for (int s = 1; s < SLICES; s++)
#pragma unroll
        for (int e = 0; e < 8; e++)
            z[e] += sums[s][lane][e];
    float b[8];
    load_bias(KIND != PLAIN ? a.e.bias : nullptr, col, count, b);
    Eight<T> other{};
    if (KIND != PLAIN && a.e.other)
        other.load(reinterpret_cast<const char *>(a.e.other) + row * a.e.other_stride + (int64_t)col * sizeof(T), count);
    RecdBits bits{};
    if (KIND != PLAIN && a.e.mask.cut)
        bits = recd_mask_bits(a.e.mask, recd_mask_call(a.e.mask), a.e.row0 + row, col >> 3);
    finish<T, KIND>(a.e, bits, row, col, count, a.n_j, b, z, other, nullptr, unit);
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

// Few rows: 16 features a block, whose waves take equal parts of the contraction (or of a split of it), straight from memory to the
// matrix cores; their sums are added up in LDS in the waves' order.  What bounds it is how many loads a compute unit has on their way: eight waves
// with sixteen of each operand (fp32: sixteen with eight) for up to 16 rows.  One row 4096 -> 4096 bf16: 9.3 us a call, sixteen waves 11.3, four
// 14.2; fp32 16.8, eight waves 20.1.
// PARTS: of at most 16 / PARTS rows and features, the matrix instruction's 16 rows and columns hold PARTS neighbouring pieces of the contraction
// each: the sums of a piece with itself count, and every load still brings 16 pieces of 64 bytes of w.
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

template <typename T, int RG, int W, int UNROLL, int PARTS = 1> __global__ __launch_bounds__(64 * W) void k_few(ProductArgs a)
{
    constexpr int FE = 16 / PARTS;  // features, and with parts rows
    static_assert(PARTS == 1 || RG == 1);
    __shared__ float join[W][16 * RG][16 + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = blockIdx.x * FE, n = (int)a.n_i, K = (int)a.K, part = (lane & 15) / FE;
    const int j = j0 + (lane & (FE - 1)) < a.n_j ? j0 + (lane & (FE - 1)) : a.n_j - 1;
    const char *q = (const char *)a.q + j * a.q_stride;
    const char *p[RG];
#pragma unroll
    for (int g = 0; g < RG; g++) {
        const int i = 16 * g + (lane & (FE - 1));
        p[g] = (const char *)a.p + (i < n ? i : n - 1) * a.p_stride;
    }
    recd_f32x4 acc[RG];
#pragma unroll
    for (int g = 0; g < RG; g++)
        acc[g] = recd_f32x4{};
    constexpr int STEP = 32 * PARTS;
    const int of_split = (int)(a.k_each / STEP), c0 = (int)blockIdx.y * of_split, each = (of_split + W - 1) / W;
    const int all = (K + STEP - 1) / STEP < c0 + of_split ? (K + STEP - 1) / STEP : c0 + of_split;
    const int c1 = c0 + (wave + 1) * each < all ? c0 + (wave + 1) * each : all;
#pragma unroll UNROLL
    for (int c = c0 + wave * each; c < c1; c++) {
        const int k = STEP * c + 32 * part + 8 * (lane >> 4);
        const auto qf = few_frag<T>(q, k, K);
#pragma unroll
        for (int g = 0; g < RG; g++)
            acc[g] = Mma16<T>::mul(qf, few_frag<T>(p[g], k, K), acc[g]);
    }
#pragma unroll
    for (int g = 0; g < RG; g++)
        *reinterpret_cast<recd_f32x4 *>(&join[wave][16 * g + (lane & 15)][4 * (lane >> 4)]) = acc[g];
    __syncthreads();
    // eight sums of a row; with four parts the block has one half of them
    const int row = PARTS == 1 ? threadIdx.x >> 1 : threadIdx.x, at = PARTS == 1 ? 8 * (threadIdx.x & 1) : 0, col = (j0 + at) & ~7;
    const int half = PARTS == 4 ? j0 >> 2 & 1 : -1;
    if (row >= (PARTS == 1 ? 16 * RG : FE) || row >= n || col >= a.n_j)
        return;
    const int count = a.n_j - col >= 8 ? 8 : a.n_j - col;
    float z[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        z[e] = 0.0f;
        if (PARTS == 4 && e >> 2 != half)
            continue;
        for (int w = 0; w < W; w++)
#pragma unroll
            for (int h = 0; h < PARTS; h++)  // (products of one part with another are for nobody)
                z[e] += join[w][row + FE * h][PARTS == 4 ? (e & 3) + 4 * h : at + 8 * h + e];
    }
    if (a.part) {
        recd_store8(a.part + ((int64_t)blockIdx.y * n + row) * a.n_j + col, count, z);
        return;
    }
    load_bias(a.e.bias, col, count, b);
    Eight<T> other{};
    if (a.e.other)
        other.load(reinterpret_cast<const char *>(a.e.other) + row * a.e.other_stride + (int64_t)col * sizeof(T), count);
    const RecdBits bits = a.e.mask.cut ? recd_mask_bits(a.e.mask, recd_mask_call(a.e.mask), a.e.row0 + row, col >> 3) : RecdBits{};
    finish<T, FORWARD>(a.e, bits, row, col, count, a.n_j, b, z, other, nullptr, 1.0f, half);
}

// ---- how a call is cut ---------------------------------------------------------------------------------------------

constexpr int kFewRows = 64;

struct Shape {
    int side, side_j;      // rows and columns of a block's tile
    int tiles_i, tiles_j, splits;
    int64_t k_each, turn;  // rows of one launch
};

// What a tile of `side` costs on a compute unit, in us: a step of the contraction, and its beginning and end, for one block alone
// (`turned`: both operands' rows run along i and j, as grad_w has them) and for each of those that share the unit (`resident` at a time).
// `heavy`: with an activation or dropout at the end.
struct Cost {
    int side, side_j, resident;
    float step_alone, step_turned, step, ends_alone, ends, ends_heavy;
};
constexpr Cost kCost16[] = {{256, 256, 1, 1.5f, 1.5f, 1.7f, 9.0f, 8.0f, 20.0f},
                            {128, 128, 2, 0.6f, 0.85f, 0.52f, 3.0f, 3.5f, 5.0f},
                            {64, 64, 4, 0.38f, 0.38f, 0.19f, 1.0f, 3.0f, 4.0f}};
constexpr Cost kCost32[] = {{128, 128, 2, 2.2f, 2.2f, 1.9f, 3.0f, 3.5f, 5.0f},
                            {64, 64, 4, 0.75f, 0.75f, 0.5f, 1.0f, 3.0f, 4.0f},
                            {128, 32, 4, 0.75f, 0.75f, 0.5f, 1.0f, 3.0f, 4.0f}};

// The tile and the number of splits of least cost: by rounds of blocks on the compute units, and with splits by the launch that adds
// them up and its traffic (8 bytes a sum at about 4.5 TB/s).  Measured (us, 16 bits; side / splits): 16 384 x 8192 -> 1024, grad_w 256/1 434,
// 256/2 283, 128/1 310, 64/1 445; 16 384 x 2048 -> 1024, grad_w 128/2 122, 128/4 82, 256/6 87; 4096 x 2048 -> 2048 256/1 53, 128/1 40,
// 64/1 52; 512 x 4096 -> 1024 256/8 31, 128/4 20, 64/1 27, 64/2 16; 128 x 8192 -> 1024 128/8 19, 64/1 55, 64/8 14.5; 300 007 x 128 -> 512
// with GELU and dropout 256/1 243, 128/1 205; 32 bits: 18 307 x 5072 -> 140 64/1 327, 128 x 32/1 295, 2000 x 2048 -> 160 64/4 27,
// 128 x 32/3 23.
Shape product_shape(const recd_ctx *ctx, int64_t n_i, int n_j, int64_t K, recd_dtype dt, bool heavy, bool turned = false)
{
    const int bk = 128 / (int)elem_size(dt);
    const int64_t steps = (K + bk - 1) / bk;
    Shape s;
    s.side = s.side_j = 64;
    int64_t splits = 1;
    double least = 1e30;
    const Cost *costs = dt == RECD_F32 ? kCost32 : kCost16, *const end = costs + 3;
    for (; costs != end; costs++) {
        const Cost &c = *costs;
        const int64_t tiles = ((n_i + c.side - 1) / c.side) * ((n_j + c.side_j - 1) / c.side_j);
        for (int64_t k = 1; k <= 256 && (k == 1 || 4 * k <= steps); k += k < 4 ? 1 : k / 2) {
            const int64_t blocks = (tiles * k + ctx->num_cu - 1) / ctx->num_cu, each = (steps + k - 1) / k;
            const double step_alone = turned ? c.step_turned : c.step_alone;
            const double alone = (double)((blocks + c.resident - 1) / c.resident) * ((double)each * step_alone + c.ends_alone);
            const double shared = (double)blocks * ((double)each * c.step + (heavy && k == 1 ? c.ends_heavy : c.ends));
            const double join = k == 1 ? 0.0 : 5.0 + (double)k * (double)n_i * n_j * 8.0 / 4.5e6;
            const double cost = (alone > shared ? alone : blocks == 1 ? alone : shared) + join;
            if (cost < least) {
                least = cost;
                splits = k;
                s.side = c.side;
                s.side_j = c.side_j;
            }
        }
    }
    const int64_t each = steps ? (steps + splits - 1) / splits : 1;
    s.k_each = each * bk;
    s.splits = (int)((steps + each - 1) / each);
    if (s.splits < 1)
        s.splits = 1;
    s.tiles_j = (n_j + s.side_j - 1) / s.side_j;
    // blocks of one launch: below 2^22
    const int64_t most = ((int64_t)1 << 22) / s.tiles_j * s.side;
    s.turn = s.splits > 1 || n_i <= most ? n_i : most;
    s.tiles_i = (int)((s.turn + s.side - 1) / s.side);
    return s;
}

// f(tile's waves and tiles of them as constants), of the tile that a shape names
template <typename T, typename F> void with_tile(const Shape &s, F f)
{
    auto tile = [&]<int WI, int WJ, int TI, int TJ>() { f.template operator()<WI, WJ, TI, TJ>(); };
    if (s.side == 256) {
        if constexpr (sizeof(T) == 2)
            tile.template operator()<2, 4, 4, 2>();
    } else if (s.side_j == 32) {
        if constexpr (sizeof(T) == 4)
            tile.template operator()<4, 1, 1, 1>();
    } else if (s.side == 128)
        tile.template operator()<2, 2, 2, 2>();
    else
        tile.template operator()<2, 2, 1, 1>();
}

unsigned product_blocks(ProductArgs &a, const Shape &s)
{
    a.tiles_i = (int)((a.n_i + s.side - 1) / s.side);
    a.tiles_j = s.tiles_j;
    a.splits = s.splits;
    a.k_each = s.k_each;
    return (unsigned)(((int64_t)a.tiles_i * a.tiles_j * a.splits + 7) / 8 * 8);
}

template <typename T, bool PCOLS, bool QCOLS, int KIND> void launch_product(ProductArgs a, const Shape &s, hipStream_t st)
{
    const int64_t n = a.n_i;
    for (int64_t i0 = 0; i0 < n; i0 += s.turn) {
        ProductArgs b = a;
        b.n_i = n - i0 < s.turn ? n - i0 : s.turn;
        b.p = (const char *)a.p + (PCOLS ? i0 * (int64_t)sizeof(T) : i0 * a.p_stride);
        if (a.e.other)
            b.e.other = (const char *)a.e.other + i0 * a.e.other_stride;
        if (a.e.out)
            b.e.out = (char *)a.e.out + i0 * a.e.out_stride;
        if (a.e.sums)
            b.e.sums = a.e.sums + i0 * a.n_j;
        if (a.e.col_part)
            b.e.col_part = a.e.col_part + i0 / s.side * a.n_j;
        b.e.row0 = a.e.row0 + i0;
        const unsigned blocks = product_blocks(b, s);
        with_tile<T>(s, [&]<int WI, int WJ, int TI, int TJ>() {
            hipLaunchKernelGGL((k_product<T, PCOLS, QCOLS, WI, WJ, TI, TJ, KIND>), dim3(blocks), dim3(64 * WI * WJ), 0, st, b);
        });
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
    if constexpr (KIND != GRAD)  // (which takes column sums besides)
        if (a.splits >= SLICES) {
            hipLaunchKernelGGL((k_join<T, KIND>), dim3((unsigned)((a.n_i * a.per_row + 63) / 64)), dim3(64 * SLICES), 0, st, a);
            return;
        }
    hipLaunchKernelGGL((k_rows<T, KIND>), dim3((unsigned)s.groups, (unsigned)s.blocks), dim3(kBlock), 0, st, a, s.clog);
}

// ---- the workspace of a pair of calls --------------------------------------------------------------------------------

struct ForwardPlan {
    bool few;
    int parts;             // of k_few
    Shape shape;
    float *part;

    void make(const recd_ctx *ctx, const recd_dense_layer *a, bool heavy, char *ws, size_t *bytes)
    {
        WsCarver c(ws);
        // The kernel of few rows reads all of them for every 16 features, the tiles' for 64 (us: 64 rows 4096 -> 4096 bf16 23 and 15, 37 rows
        // 512 -> 128 fp32 7.3 and 9.5).  Few features leave most of the card idle: then the contraction is split, if it is long
        few = a->n <= 16 || (a->n <= kFewRows && a->in <= 512);
        part = nullptr;
        if (few) {
            const int64_t chunks = (a->in + 31) / 32, blocks = (a->out + 15) / 16;
            int64_t splits = ctx->num_cu / blocks < chunks / 32 ? ctx->num_cu / blocks : chunks / 32;
            splits = splits < 1 ? 1 : splits > 8 ? 8 : splits;
            const int64_t each = (chunks + splits - 1) / splits;
            shape.k_each = 32 * each;
            shape.splits = (int)((chunks + each - 1) / each);
            // Blocks of fewer features in place of splits and the launch that adds them up, up to 64 KiB of w a block, which a unit fetches in
            // about 5 us (us a call, splits and parts: one row 4096 -> 1024 bf16 10.4 and 6.8, 8192 -> 1024 11.2 and 9.3, eight rows,
            // 128 KiB, 12.1 and 13.6); without splits for long rows of 16 bits (one row 8192 -> 4096 22.3 and 16.3, 1024 -> 8192 7.1 and 9.1, fp32
            // 2048 -> 4096 9.4 and 14.3)
            const int row_bytes = a->in * (int)elem_size(a->dtype);
            parts = a->n <= 4 ? 4 : a->n <= 8 ? 2 : 1;
            if (row_bytes > (1 << 12) * parts || (shape.splits == 1 && (a->dtype == RECD_F32 || a->in < 4096)))
                parts = 1;
            if (parts > 1) {
                shape.k_each = (a->in + 32 * parts - 1) / (32 * parts) * (32 * parts);
                shape.splits = 1;
            }
        } else
            shape = product_shape(ctx, a->n, a->out, a->in, a->dtype, heavy);
        if (shape.splits > 1)
            part = c.take<float>((size_t)shape.splits * a->n * a->out);
        *bytes = c.off;
    }
};

struct BackwardPlan {
    bool need_gz, again;   // gz differs from grad_y; z is made again
    Shape z, gx, gw;
    int64_t col_blocks;
    char *gz;
    uint32_t *largest;     // of k_largest, where gz is of fp16
    float *unit;
    bool together;         // the gradients of x and w go into one launch
    float *part, *part_w, *col_part;  // (z's and grad_x's parts in turn; grad_w's)

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
        const bool scaled = need_gz && (grad_x || grad_w) && a->dtype == RECD_F16;
        largest = scaled ? c.take<uint32_t>(kLargest) : nullptr;
        unit = scaled ? c.take<float>(1) : nullptr;
        size_t parts = 0, parts_w = 0;
        if (again) {
            z = product_shape(ctx, a->n, a->out, a->in, a->dtype, true);
            if (z.splits > 1)
                parts = larger(parts, (size_t)z.splits * a->n * a->out);
        }
        if (grad_x) {
            gx = product_shape(ctx, a->n, a->in, a->out, a->dtype, false);
            if (gx.splits > 1)
                parts = larger(parts, (size_t)gx.splits * a->n * a->in);
        }
        if (grad_w) {
            gw = product_shape(ctx, a->out, a->in, a->n, a->dtype, false, true);
            if (gw.splits > 1)
                parts_w = (size_t)gw.splits * a->out * a->in;
        }
        together = grad_x && grad_w && gx.side == gw.side && gx.side_j == gw.side_j && gx.side < 256 && gx.turn == a->n;
        if (!together) {
            parts = larger(parts, parts_w);
            part = part_w = parts ? c.take<float>(parts) : nullptr;
        } else {
            part = parts ? c.take<float>(parts) : nullptr;
            part_w = parts_w ? c.take<float>(parts_w) : nullptr;
        }
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
    if ((uintptr_t)p % 16 || stride < width || stride >= ((int64_t)1 << 24) / e || stride * e % 16)
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
    ForwardPlan().make(&c, sizes, sizes->act != RECD_ACT_NONE || mask.cut, nullptr, &forward);
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
    plan.make(ctx, a, a->act != RECD_ACT_NONE || mask.cut, nullptr, &bytes);
    if (bytes) {
        ctx->plan.valid = false;  // the parts overwrite the workspace a backward plan would live in
        RECD_TRY(recd_reserve(ctx, bytes));
        plan.make(ctx, a, a->act != RECD_ACT_NONE || mask.cut, ctx->ws, &bytes);
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
    p.e = Epilogue{(int)a->act, mask, 0, bias, residual, a->residual_stride * e, y, a->y_stride * e, sums, nullptr, nullptr, nullptr};
    recd_with_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        if (plan.few) {
            const int features = 16 / plan.parts;
            const dim3 grid((unsigned)((a->out + features - 1) / features), (unsigned)plan.shape.splits);
            constexpr int W = sizeof(T) == 4 ? 16 : 8;
            p.k_each = plan.shape.k_each;
            if (plan.parts == 4)
                hipLaunchKernelGGL((k_few<T, 1, W, 128 / W, 4>), grid, dim3(64 * W), 0, ctx->stream, p);
            else if (plan.parts == 2)
                hipLaunchKernelGGL((k_few<T, 1, W, 128 / W, 2>), grid, dim3(64 * W), 0, ctx->stream, p);
            else if (a->n <= 16)
                hipLaunchKernelGGL((k_few<T, 1, W, 128 / W>), grid, dim3(64 * W), 0, ctx->stream, p);
            else if (a->n <= 32)
                hipLaunchKernelGGL((k_few<T, 2, 8, 4>), grid, dim3(64 * 8), 0, ctx->stream, p);
            else
                hipLaunchKernelGGL((k_few<T, 4, 8, 4>), grid, dim3(64 * 8), 0, ctx->stream, p);
        } else
            launch_product<T, false, false, FORWARD>(p, plan.shape, ctx->stream);
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
        Epilogue ep{(int)a->act, mask, 0, bias, grad_y, grad_y_stride * e, plan.gz, out * e, nullptr, plan.col_part, plan.largest, plan.unit};
        if (plan.largest)
            hipLaunchKernelGGL(k_largest, dim3(kLargest), dim3(1024), 0, st, a->n, out / 8, (const char *)grad_y, grad_y_stride * e,
                               plan.largest);
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
                launch_product<T, false, false, GRAD>(p, plan.z, st);
            }
            if (!plan.again || plan.z.splits > 1) {
                RowsArgs r{a->n, out, 0, plan.again ? plan.z.splits : 1, plan.again ? plan.part : nullptr, plan.again ? nullptr : sums, 0, ep};
                if (r.parts && r.splits >= 2 * SLICES) {
                    // their sum first, in the first one's place (27 rows 5844 -> 60 fp32 with SiLU: gz and grad_bias 23.4 us without, 16.3 with
                    // it; from eight splits on 64 rows 4096 -> 128 bf16 13.8 and 16.7)
                    RowsArgs z = r;
                    z.e = Epilogue{};
                    z.e.out = plan.part;
                    z.e.out_stride = out * (int64_t)sizeof(float);
                    launch_rows<float, PLAIN>(ctx, z, st);
                    r.splits = 1;
                }
                launch_rows<T, GRAD>(ctx, r, st);
            }
        }
        if (grad_bias)
            hipLaunchKernelGGL(k_join_columns, dim3((unsigned)((out + 31) / 32)), dim3(1024), 0, st, plan.col_blocks, out,
                               plan.col_part, grad_bias);
        ProductArgs px{}, pw{};
        px.n_i = a->n;
        px.n_j = in;
        px.K = out;
        px.p = gz;
        px.q = w;
        px.p_stride = gz_stride;
        px.q_stride = in * e;
        px.part = a->n > 0 && grad_x && plan.gx.splits > 1 ? plan.part : nullptr;
        px.e.out = grad_x;
        px.e.out_stride = grad_x_stride * e;
        px.e.unit = pw.e.unit = plan.unit;
        pw.n_i = out;
        pw.n_j = in;
        pw.K = a->n;
        pw.p = gz;
        pw.q = x;
        pw.p_stride = gz_stride;
        pw.q_stride = a->x_stride * e;
        pw.part = grad_w && plan.gw.splits > 1 ? plan.part_w : nullptr;
        pw.e.out = grad_w;
        pw.e.out_stride = in * e;
        if (plan.together) {
            const unsigned blocks_w = product_blocks(pw, plan.gw), blocks_x = product_blocks(px, plan.gx);
            with_tile<T>(plan.gx, [&]<int WI, int WJ, int TI, int TJ>() {
                if constexpr (32 * WI * TI < 256)
                    hipLaunchKernelGGL((k_gradients<T, WI, WJ, TI, TJ>), dim3(blocks_w + blocks_x), dim3(64 * WI * WJ), 0, st, px, pw, blocks_w);
            });
        } else {
            if (a->n > 0 && grad_x)
                launch_product<T, false, true, PLAIN>(px, plan.gx, st);
            if (px.part)  // (its place is grad_w's too)
                launch_rows<T, PLAIN>(ctx, RowsArgs{a->n, in, 0, plan.gx.splits, px.part, nullptr, 0, px.e}, st);
            if (grad_w)
                launch_product<T, true, true, PLAIN>(pw, plan.gw, st);
        }
        if (plan.together && px.part)
            launch_rows<T, PLAIN>(ctx, RowsArgs{a->n, in, 0, plan.gx.splits, px.part, nullptr, 0, px.e}, st);
        if (pw.part)
            launch_rows<T, PLAIN>(ctx, RowsArgs{out, in, 0, plan.gw.splits, pw.part, nullptr, 0, pw.e}, st);
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

} // extern "C"
