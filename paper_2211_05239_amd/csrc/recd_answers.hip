// Answers of rows x [n, D] scored against a whole table [V, D]: sum of the softmax and its entropy, the log probability of a given
// id, and the k most likely ids.
//
//   z_iv = scale * x_i . W_v,  lse_i = log sum_v exp(z_iv),  logp_i = z_i,given(i) - lse_i
//   H_i = -sum_v p_iv log p_iv = log s + t / s  with  s = sum_v exp(z_iv - m),  t = sum_v exp(z_iv - m) (m - z_iv)
//
// The logits [n, V] are never stored.  The first kernel streams the table once past rows that stay in registers, with a running
// maximum m, s and t per row, and writes the largest logit of every chunk of 64 table rows.  The k best ids lie in chunks whose
// largest logit is among the k best ones' (to the error of 32 bits): the second kernel finds these few chunks for each
// row and computes their logits again, in 64 bits, which puts neighbours in rank in order that 32 bits do not tell apart.
// Both terms of H are at least 0, so nothing cancels where one id has nearly all of the weight.
//
// What bounds them.  Many rows: the vector units.  A logit takes the matrix cores 2 D operations, and the vector units about seven instructions:
// the product with scale, half a maximum, the exponential (twice the time of another), the two sums.  4096 rows of 1 M x 128 bf16 take 1600 to 1700
// us, the clock's share in it, 0.65 PFLOP/s beside a large product's 1.40: 1430 at least in the first kernel, which has the vector units 67 % busy
// and the matrix cores 33 %, its waves waiting 43 % of their time (each at the exchange of its pairs' maxima, before its exponentials); 230 in the
// second, which is bound by memory: the chunks' maxima twice and the listed chunks, 1.09 GB at 4.8 TB/s.  Few rows: the table's way from
// memory, 1 M x 128 bf16 at 5.5 TB/s (46 us for one row without ids), and for small tables the two launches and the chains of their loads (37 rows of
// 100 000 x 64 fp32: 17 and 15 us).  More ids than a table has chunks: all of it is computed again in 64 bits, and put in order a
// thousand at a time (4096 rows of 2000 x 64 bf16 with 64 ids: 266 us).
#include "recd_internal.h"
#include "recd_mfma.h"

#include <math.h>

namespace {

constexpr int kChunk = 64;       // table rows
constexpr int kWaves = 4;        // of the kernel of few rows
constexpr int kMany = 8;         // of the kernel of many rows
constexpr int kFewRows = 256;   // of 300 000 x 128 bf16, eight ids: 256 rows 73 us here, 300 rows by the kernel of many 96

struct StreamArgs {
    int64_t n, V;
    int D;
    float c;             // |scale| * log2(e); the sign goes into the kept side
    bool negative;
    const void *x, *table;
    int row_blocks, splits;
    int64_t chunks, each;            // chunks of a split (a multiple of 4 in the kernel of many rows)
    float *part_m, *part_s, *part_t; // [splits][n], in powers of two
    float *best;                     // [n][stride]: the chunks' largest logits, or null
    int64_t stride;
    uint32_t *widest;                // [chunks]: the largest absolute value in a chunk's table rows, as an integer, or null
};

// The larger of `top` and the absolute values in a piece: of 16-bit values in both halves.
template <typename T> __device__ inline uint32_t widest_of(uint32_t top, typename RecdPiece<T>::type piece)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const recd_u32x4 b = __builtin_bit_cast(recd_u32x4, piece);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (sizeof(T) == 4)
            top = max(top, b[i] & 0x7fffffffu);
        else
            top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                                        __builtin_bit_cast(u16x2, b[i] & 0x7fff7fffu)));
    }
    return top;
}

// The wave's largest, without a way through LDS: neighbours, then rows of 16 lanes, then these to the next ones.
__device__ inline uint32_t wave_top(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));   // lanes ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));   // lanes ^ 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));  // mirrored in eight
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));  // mirrored in sixteen
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false)); // lane 15 of a row to the next
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false)); // lane 31 to the upper half
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// The wave's largest, as the bits of a float.
template <typename T> __device__ inline uint32_t widest_float(uint32_t top)
{
    if constexpr (sizeof(T) == 2) {
        const uint32_t a = top & 0xffffu, b = top >> 16, both = a > b ? a : b;
        top = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(T, (unsigned short)both)) & 0x7fffffffu;  // (a NaN's is above an infinity's)
    }
    return wave_top(top);
}

struct Running {
    float m = -INFINITY, s = 0.0f, t = 0.0f;  // maximum (in powers of two), sum of e, sum of e * log2(e)

    __device__ inline void rescale(float top)
    {
        const float now = fmaxf(m, top);
        if (now == m)
            return;
        // (m = -inf: nothing has been added up)
        const float f = m == -INFINITY ? 0.0f : recd_exp2(m - now), by = m == -INFINITY ? 0.0f : m - now;
        t = (t + s * by) * f;
        s *= f;
        m = now;
    }
    __device__ inline void join(float om, float os, float ot)
    {
        rescale(om);
        if (om == -INFINITY)
            return;
        const float f = recd_exp2(om - m);
        t += (ot + os * (om - m)) * f;
        s += os * f;
    }
};

// The same of one lane along its part of the table, with sums whose loss does not grow with it: sixteen scores at a time are added up in 32
// bits behind the maximum, and their sums in 64 bits behind the whole number next to it, so that a move to a larger maximum only
// multiplies by a power of two; every score is rounded by one factor, whatever moves come after it.  (With 32-bit sums that every score was added
// to, one logit over a million equal ones left lse off by 0.018 where 131 072 rows take the table in one split, a thousand times what
// the logits' own roundings leave.)  t stays behind the maximum itself, as it would cancel against log s otherwise.
struct Along {
    float m = -INFINITY, unit = 1.0f;  // 2^(m - rint(m)), which s and t are to be divided by
    double s = 0.0, t = 0.0;

    // The sums move by what the maximum does as it is held, that is rounded: 0 in the last digits of a large one, where the scores' own
    // difference to it may still be anything.
    __device__ inline void move(float now)
    {
        const int shift = (int)fminf(fmaxf(rintf(m) - rintf(now), -2000.0f), 0.0f);
        const double by = m == -INFINITY ? 0.0 : (double)(m - now);  // (of a first one nothing has been added up)
        t = ldexp(fma(s, by, t), shift);
        s = ldexp(s, shift);
        unit = recd_exp2(now - rintf(now));
        m = now;
    }
    __device__ inline void add(float ds, float dt)
    {
        s += (double)(ds * unit);
        t += (double)(dt * unit);
    }
};

// Below this a sum of absolute products leaves 32-bit sums finite, in whatever order, and the logits in powers of two too.
constexpr float kReach = 4e37f;

// Scores of 32 table rows, half of them in each lane of a pair, into the running sums; `left` of these rows are there.  Returns the
// largest logit in powers of two.  It is found among what the exponentials are taken of anyway, z * c - m: the maximum of the scores
// themselves would take an operation more for each.  Behind the table's end stand scores of one of its rows over again (its last one's),
// which leave the maximum as it is; only the sums leave them out.  Behind an infinite logit the maximum starts again: the sums are NaN for
// good, but the chunks' largest logits are still asked for.
__device__ inline float add_up(Along &run, recd_f32x16 z, float c, int left, int lane)
{
    const float from = __builtin_isinf(run.m) ? 0.0f : run.m;
#pragma unroll
    for (int r = 0; r < 16; r++)
        z[r] = __builtin_fmaf(z[r], c, -from);
    float top = -INFINITY;  // (of nothing but NaN)
#pragma unroll
    for (int r = 0; r < 16; r += 2)
        top = fmaxf(fmaxf(top, z[r]), z[r + 1]);
    top = fmaxf(top, __shfl_xor(top, 32));
    const bool moves = (top > 0.0f || run.m == -INFINITY) && top > -INFINITY && left > 0;
    auto exponentials = [&](auto moved, auto ends, float by) {
        float s = 0.0f, t = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; r++) {
            float d = moved.value ? z[r] + by : z[r];
            if (ends.value)
                d = recd_score_row(r, lane) < left ? d : -1000.0f;  // (whose exponential is 0)
            const float e = recd_exp2(d);
            s += e;
            t = __builtin_fmaf(e, d, t);
        }
        run.add(s, t);
    };
    // (maxima move seldom; all ways have exponentials of their own, or the others would copy all scores)
    if (__any(moves) || left < 32) {
        if (moves)
            run.move(from + top);
        const float by = moves ? -top : 0.0f;
        if (left < 32)
            exponentials(std::true_type{}, std::true_type{}, by);
        else
            exponentials(std::true_type{}, std::false_type{}, by);
    } else
        exponentials(std::false_type{}, std::false_type{}, 0.0f);
    return left > 0 ? from + top : -INFINITY;
}

template <typename T, int KS>
__device__ inline void keep_rows(typename RecdMma<T>::Frag (&xf)[KS], const StreamArgs &a, int64_t row, int lane)
{
#pragma unroll
    for (int k = 0; k < KS; k++) {
        xf[k] = recd_row_frag<T>((const T *)a.x + row * a.D, 16 * k, a.D, row < a.n, lane);
        if (a.negative)
            xf[k] = recd_negated(xf[k]);
    }
}

// Few rows: the block's waves hold the same 32 * N rows and each streams chunks of its own through LDS of its own.
template <typename T, int DP, int N> __global__ __launch_bounds__(64 * kWaves) void k_answers_few(StreamArgs a)
{
    constexpr int KS = DP / 16;
    using Frag = typename RecdMma<T>::Frag;
    __shared__ union {
        RecdTile<T, 32, DP> tile[kWaves];
        float join[kWaves][3][32 * N];
    } lds;
    const int rb = blockIdx.x % a.row_blocks, split = blockIdx.x / a.row_blocks;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = (int64_t)rb * 32 * N;
    const int64_t c1 = (split + 1) * a.each < a.chunks ? (split + 1) * a.each : a.chunks;
    RecdTile<T, 32, DP> &tile = lds.tile[wave];
    Frag xf[N][KS];
#pragma unroll
    for (int j = 0; j < N; j++)
        keep_rows<T, KS>(xf[j], a, row0 + 32 * j + (lane & 31), lane);
    Along run[N];
    RecdStream<T, 32, DP, 64> stream;
    if (a.D < DP)
        stream.clear_behind(lane, tile, a.D);
    // half h of chunk c; one behind the table's end is the last row over again
    auto load = [&](int64_t c, int h) {
        const int64_t first = c * kChunk + 32 * h, from = first < a.V ? first : a.V - 1;
        stream.load_rows(lane, (const T *)a.table + from * a.D, a.V - from < 32 ? (int)(a.V - from) : 32, a.D, a.D * sizeof(T));
    };
    int64_t c = split * a.each + wave;
    if (c < c1)
        load(c, 0);
    for (; c < c1; c += kWaves) {
        const int left = a.V - c * kChunk < kChunk ? (int)(a.V - c * kChunk) : kChunk;
        float top[N];
        uint32_t top_abs = 0;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            recd_wave_sync();
            stream.store(lane, tile, a.D);
            if (rb == 0 && a.widest)
#pragma unroll
                for (auto &piece : stream.held)
                    top_abs = widest_of<T>(top_abs, piece);
            recd_wave_sync();
            if (h == 0)
                load(c, 1);
            else if (c + kWaves < c1)
                load(c + kWaves, 0);
            recd_f32x16 z[N];
#pragma unroll
            for (int j = 0; j < N; j++)
                z[j] = recd_f32x16{};
#pragma unroll
            for (int k = 0; k < KS; k++) {
                const Frag w = tile.rows(0, 16 * k, lane);
#pragma unroll
                for (int j = 0; j < N; j++)
                    z[j] = RecdMma<T>::mul(w, xf[j][k], z[j]);
            }
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float half = add_up(run[j], z[j], a.c, left - 32 * h, lane);
                top[j] = h ? fmaxf(top[j], half) : half;
            }
        }
#pragma unroll
        for (int j = 0; j < N; j++) {
            const int64_t row = row0 + 32 * j + (lane & 31);
            if (a.best && lane < 32 && row < a.n)
                a.best[row * a.stride + c] = top[j] * kRecdLn2;
        }
        if (rb == 0 && a.widest) {
            top_abs = widest_float<T>(top_abs);
            if (lane == 0)
                a.widest[c] = top_abs;
        }
    }
    // the waves' sums in their order
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; j++) {
        run[j].s += __shfl_xor(run[j].s, 32);
        run[j].t += __shfl_xor(run[j].t, 32);
        if (lane < 32) {
            lds.join[wave][0][32 * j + lane] = run[j].m;
            lds.join[wave][1][32 * j + lane] = (float)(run[j].s / run[j].unit);
            lds.join[wave][2][32 * j + lane] = (float)(run[j].t / run[j].unit);
        }
    }
    __syncthreads();
    const int i = threadIdx.x;
    if (i >= 32 * N || row0 + i >= a.n)
        return;
    Running all;
    for (int w = 0; w < kWaves; w++)
        all.join(lds.join[w][0][i], lds.join[w][1][i], lds.join[w][2][i]);
    a.part_m[split * a.n + row0 + i] = all.m;
    a.part_s[split * a.n + row0 + i] = all.s;
    a.part_t[split * a.n + row0 + i] = all.t;
}

// Many rows: 32 in every wave of a block, all of which see every table row of the split, a chunk of them at a time in two
// buffers of LDS.  Four waves a SIMD for 16-bit rows of up to 128 (the stream of 4096 rows of 1 M x 128 bf16, when
// its sums were of 32 bits: 1370 us; of the compiler's own choice of three 1530, of five 1480, of six 1770).
template <typename T, int DP> __global__ __launch_bounds__(64 * kMany, sizeof(T) == 2 && DP <= 128 ? 4 : 2) void k_answers_many(StreamArgs a)
{
    constexpr int KS = DP / 16;
    using Frag = typename RecdMma<T>::Frag;
    __shared__ RecdTile<T, kChunk, DP> tiles[2];
    __shared__ uint32_t tops[2][kMany];
    // the row blocks of one split side by side on one die, whose L2 then serves the split's rows to all of them
    const int64_t total = (int64_t)a.splits * a.row_blocks, share = (total + 7) / 8;
    const int64_t at = (int64_t)(blockIdx.x & 7) * share + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= share || at >= total)
        return;
    const int split = (int)(at / a.row_blocks), rb = (int)(at - (int64_t)split * a.row_blocks);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = ((int64_t)rb * kMany + wave) * 32 + (lane & 31);
    const int64_t c0 = split * a.each, c1 = c0 + a.each < a.chunks ? c0 + a.each : a.chunks;
    Frag xf[KS];
    keep_rows<T, KS>(xf, a, row, lane);
    Along run;
    RecdStream<T, kChunk, DP, 64 * kMany> stream;
    if (a.D < DP)
        for (auto &tile : tiles)
            stream.clear_behind(tid, tile, a.D);
    auto load = [&](int64_t c) {
        const int64_t left = a.V - c * kChunk;
        stream.load_rows(tid, (const T *)a.table + c * kChunk * a.D, left < kChunk ? (int)left : kChunk, a.D, a.D * sizeof(T));
    };
    // the blocks of a split's rows find the chunks' largest values in turns: this one's is `turn` chunks away
    int turn = a.widest ? rb : INT32_MAX;
    auto store = [&](int buf, int turn) {
        stream.store(tid, tiles[buf], a.D);
        if (turn == 0) {
            uint32_t top_abs = 0;
#pragma unroll
            for (int i = 0; i < stream.PT; i++)
                if (tid + i * 64 * kMany < RecdTile<T, kChunk, DP>::PIECES)
                    top_abs = widest_of<T>(top_abs, stream.held[i]);
            top_abs = widest_float<T>(top_abs);
            if (lane == 0)
                tops[buf][wave] = top_abs;
        }
    };
    if (c0 < c1) {
        load(c0);
        store(0, turn);
        if (c0 + 1 < c1)
            load(c0 + 1);
    }
    __syncthreads();
    recd_f32x4 four = {};
    for (int64_t c = c0; c < c1; c++) {
        const int buf = (int)(c - c0) & 1;
        const int next = turn ? turn - 1 : a.row_blocks - 1;
        if (c + 1 < c1) {
            store(1 - buf, next);
            if (c + 2 < c1)
                load(c + 2);
        }
        if (turn == 0 && wave == 0) {
            const uint32_t top_abs = wave_top(lane < kMany ? tops[buf][lane] : 0);
            if (lane == 0)
                a.widest[c] = top_abs;
        }
        turn = next;
        const int left = a.V - c * kChunk < kChunk ? (int)(a.V - c * kChunk) : kChunk;
        float top = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            recd_f32x16 z = {};
#pragma unroll
            for (int k = 0; k < KS; k++)
                z = RecdMma<T>::mul(tiles[buf].rows(32 * h, 16 * k, lane), xf[k], z);
            top = fmaxf(top, add_up(run, z, a.c, left - 32 * h, lane));
        }
        if (a.best) {
            four = recd_f32x4{four[1], four[2], four[3], top * kRecdLn2};
            if ((c & 3) == 3 || c + 1 == c1) {
                for (int64_t i = c; (i & 3) != 3; i++)
                    four = recd_f32x4{four[1], four[2], four[3], -INFINITY};
                if (lane < 32 && row < a.n)
                    *reinterpret_cast<recd_f32x4 *>(a.best + row * a.stride + (c & ~(int64_t)3)) = four;
            }
        }
        __syncthreads();
    }
    run.s += __shfl_xor(run.s, 32);
    run.t += __shfl_xor(run.t, 32);
    if (lane < 32 && row < a.n) {
        a.part_m[split * a.n + row] = run.m;
        a.part_s[split * a.n + row] = (float)(run.s / run.unit);
        a.part_t[split * a.n + row] = (float)(run.t / run.unit);
    }
}

struct SelectArgs {
    int64_t n, V;
    int D, k, splits;
    float scale;
    const void *x, *table;
    const int64_t *given;
    const float *part_m, *part_s, *part_t, *best;
    const uint32_t *widest;
    int64_t chunks, stride;
    float *logp, *entropy, *lse, *top_logp;
    int64_t *top_ids;
};

constexpr int kGroups = 256, kListed = 1024;

// `a` before `b` in the answers' order.
__device__ inline bool before(double za, uint32_t a, double zb, uint32_t b) { return za > zb || (za == zb && a < b); }

// A block a row.  Let d be what a 32-bit logit of a chunk may be off by, which goes by the largest value in the chunk, so that a row of large
// values widens its own chunk alone.  At least k logits are as large as the k-th largest, L, of what the 256 groups' chunks have for
// certain, their largest logit less d: so the k best stand in chunks whose largest one and d reach L.  The logits of these chunks are
// computed again, a row of the table by neighbouring lanes, in an order that is the same for all rows, and what reaches L is kept.  Where there is no
// more room the k best of it stay, the last of which is the new bar.
template <typename T, int NT> __global__ __launch_bounds__(NT) void k_answers_select(SelectArgs a, int llog)
{
    constexpr int WAVES = NT / 64, E = 16 / sizeof(T), KEPT = 2 * WAVES * kChunk < 1024 ? 1024 : 2 * WAVES * kChunk;
    using Piece = typename RecdPiece<T>::type;
    __shared__ double key[KEPT];
    __shared__ uint32_t id[KEPT], list[kListed];
    __shared__ float groups[NT];
    __shared__ double lse_all;
    __shared__ float group_bar;
    __shared__ uint32_t count, listed, taken, top_abs[WAVES];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const T *xr = (const T *)a.x + row * a.D, *table = (const T *)a.table;
    // the lane's piece of a row, and of x: products of two of them are exact in 64 bits
    const int at = lane & ((1 << llog) - 1);
    const bool has_piece = at * E < a.D;
    double x[E];
#pragma unroll
    for (int e = 0; e < E; e++)
        x[e] = 0.0;
    if (has_piece) {
        float v[E];
        recd_load16(xr + at * E, v);
#pragma unroll
        for (int e = 0; e < E; e++)
            x[e] = (double)v[e];
    }
    auto part = [&](const Piece &v) {
        double z = 0.0;
#pragma unroll
        for (int e = 0; e < E; e++)
            z = fma(x[e], (double)(float)v[e], z);
        return z;
    };
    // what does not depend on the chunks, by one wave: the splits' sums, a lane's in their order, then the lanes'; the given id
    auto rest = [&] {
        Running all;
#pragma unroll 4
        for (int s = lane; s < a.splits; s += 64)
            all.join(a.part_m[s * a.n + row], a.part_s[s * a.n + row], a.part_t[s * a.n + row]);
        for (int o = 1; o < 64; o <<= 1) {
            const float m = __shfl_down(all.m, o), s = __shfl_down(all.s, o), t = __shfl_down(all.t, o);
            if ((lane & (2 * o - 1)) == 0)
                all.join(m, s, t);
        }
        const double lse = (double)all.m * 0.6931471805599453 + log((double)all.s);
        if (lane == 0) {
            lse_all = lse;
            if (a.lse)
                a.lse[row] = (float)lse;
            if (a.entropy)
                a.entropy[row] = (float)(log((double)all.s) - 0.6931471805599453 * (double)all.t / (double)all.s);
        }
        if (!a.given)
            return;
        const int64_t g = a.given[row];
        const bool has = g >= 0 && g < a.V;
        Piece v{};
        if (has && has_piece)
            v = *reinterpret_cast<const Piece *>(table + g * a.D + at * E);
        double z = part(v);
        for (int o = 1; o < 1 << llog; o <<= 1)
            z += __shfl_xor(z, o);
        if (lane == 0)
            a.logp[row] = has ? (float)(z * (double)a.scale - lse) : 0.0f;
    };
    if (a.k == 0) {
        if (wave == 0)
            rest();
        return;
    }
    if (NT == 256 && wave == WAVES - 1)
        rest();
    // 2^-22 of the largest sum of absolute products for each step of the sum, and what each loses where it underflows
    float sum_x = 0.0f;
#pragma unroll
    for (int e = 0; e < E; e++)
        sum_x += fabsf((float)x[e]);
    for (int o = 1; o < 1 << llog; o <<= 1)
        sum_x += __shfl_xor(sum_x, o);
    const float reach = sum_x * fmaxf(1.0f, fabsf(a.scale)), by_wide = (float)(a.D + 8) * (0x1p-22f * fabsf(a.scale) * sum_x);
    const float underflow = (float)(a.D + 8) * (2e-38f * fmaxf(1.0f, fabsf(a.scale)));
    auto off = [&](uint32_t wide) {
        const float w = __builtin_bit_cast(float, wide);
        return sum_x != 0.0f && w != 0.0f && reach * w < kReach ? by_wide * w + underflow : 0.0f;
    };
    // the groups' largest chunks: every 256th one
    const float *best = a.best + row * a.stride;
    float top = -INFINITY;
    uint32_t wide = 0;
#pragma unroll 8
    for (int64_t c = tid; c < a.chunks; c += NT) {
        const uint32_t w = a.widest[c];
        top = fmaxf(top, best[c] - off(w));
        wide = max(wide, w);
    }
    groups[tid] = top;
    wide = wave_top(wide);
    if (lane == 0)
        top_abs[wave] = wide;
    if (tid == 0)
        count = 0;
    __syncthreads();
    if (wave == 0) {
        // the k-th largest of the groups, bit by bit, of integers in the floats' order
        constexpr int MINE = kGroups / 64;
        uint32_t g[MINE];
#pragma unroll
        for (int i = 0; i < MINE; i++) {
            float top = -INFINITY;
            for (int n = lane + 64 * i; n < NT; n += kGroups)
                top = fmaxf(top, groups[n]);
            const uint32_t b = __builtin_bit_cast(uint32_t, top);
            g[i] = b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
        }
        uint32_t bar = 0;
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
            int reach = 0;
#pragma unroll
            for (int i = 0; i < MINE; i++)
                reach += __popcll(__ballot(g[i] >= (bar | bit)));
            if (reach >= a.k)
                bar |= bit;
        }
        if (lane == 0)
            group_bar = __builtin_bit_cast(float, bar ^ (bar >> 31 ? 0x80000000u : 0xffffffffu));
    }
    for (int i = 0; i < WAVES; i++)
        wide = max(wide, top_abs[i]);
    // without a bound, where the sum is not finite or could pass the range, the chunks are those that 32 bits name, and the best of them are kept
    const bool bound = reach * __builtin_bit_cast(float, wide) < kReach;
    __syncthreads();
    // what is kept comes before (bar, bar_id): the smallest of the k best so far, or all that may be among them
    const double chunk_bar = group_bar;
    double bar = bound ? chunk_bar : -INFINITY;
    uint32_t bar_id = 0xffffffffu;
    auto may_hold = [&](int64_t c) {
        const double v = (double)best[c] + (double)off(a.widest[c]);
        return v >= chunk_bar && (v > bar || (v == bar && (uint64_t)c * kChunk < bar_id));
    };
    auto ranked = [&](int kept) {
        if (kept >= a.k) {
            bar = key[a.k - 1];
            bar_id = id[a.k - 1];
        }
        if (tid == 0)
            count = kept < a.k ? kept : a.k;
        __syncthreads();
    };
    // what is kept, in order; of more than k the k best
    auto settle = [&] {
        const int kept = (int)count;
        if (kept <= NT) {  // a thread's place is the number of those before it
            const double z = tid < kept ? key[tid] : 0.0;
            const uint32_t v = tid < kept ? id[tid] : 0;
            int place = 0;
            if (tid < kept)
                for (int i = 0; i < kept; i++)
                    place += before(key[i], id[i], z, v);
            __syncthreads();
            if (tid < kept) {
                key[place] = z;
                id[place] = v;
            }
            __syncthreads();
            ranked(kept);
            return;
        }
        int size = 2;
        while (size < kept)
            size <<= 1;
        for (int i = kept + tid; i < size; i += NT) {
            key[i] = -INFINITY;
            id[i] = 0xffffffffu;
        }
        __syncthreads();
        for (int run = 2; run <= size; run <<= 1)
            for (int o = run >> 1; o; o >>= 1) {
                for (int i = tid; i < size >> 1; i += NT) {
                    const int p = (i & ~(o - 1)) << 1 | (i & (o - 1)), q = p | o;
                    const double zp = key[p], zq = key[q];
                    const uint32_t ip = id[p], iq = id[q];
                    if (before(zq, iq, zp, ip) == ((p & run) == 0)) {
                        key[p] = zq;
                        key[q] = zp;
                        id[p] = iq;
                        id[q] = ip;
                    }
                }
                __syncthreads();
            }
        ranked(kept);
    };
    // the chunk's logits, by the wave: eight loads at a time of as many table rows as the lanes hold.  Their lanes' parts are added up
    // in one tree for all of them: at each of its first steps a lane hands half of the sums to its neighbour and takes the other half
    // over, so that at the end every lane has sums of its own
    auto logits = [&](int64_t chunk) {
        const int per = 64 >> llog;  // table rows of a load
        for (int r = 0; r < kChunk; r += 8 * per) {
            Piece v[8];
            const uint32_t first = (uint32_t)(chunk * kChunk) + (uint32_t)(r + (lane >> llog));
#pragma unroll
            for (int i = 0; i < 8; i++) {
                v[i] = Piece{};
                if (has_piece && r + i * per < kChunk && first + i * per < a.V)
                    v[i] = *reinterpret_cast<const Piece *>(table + (int64_t)(first + i * per) * a.D + at * E);
            }
            double z[8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                z[i] = part(v[i]);
            int have = 8, mine = 0;  // sums of the lane, and which load's the first of them is
#pragma unroll
            for (int step = 0; step < 3; step++)
                if (step < llog) {
                    const int o = 1 << step, half = 4 >> step;
                    const bool upper = lane & o;
#pragma unroll
                    for (int i = 0; i < half; i++) {
                        const double give = upper ? z[i] : z[i + half], keep = upper ? z[i + half] : z[i];
                        z[i] = keep + __shfl_xor(give, o);
                    }
                    have = half;
                    mine += upper ? half : 0;
                }
            for (int o = 8; o < 1 << llog; o <<= 1)
                z[0] += __shfl_xor(z[0], o);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int load = mine + i;
                const uint32_t v = first + load * per;
                double s = z[i] * (double)a.scale;
                s = s == s ? s : -INFINITY;
                if (i < have && at < 8 && r + load * per < kChunk && v < a.V && before(s, v, bar, bar_id)) {
                    const uint32_t slot = atomicAdd(&count, 1u);
                    key[slot] = s;
                    id[slot] = v;
                }
            }
        }
    };
    int64_t range = a.chunks;  // chunks that are listed at a time: all, or where these are too many, as many as there is room for
    for (int64_t from = 0; from < a.chunks;) {
        const int64_t to = a.chunks - from < range ? a.chunks : from + range;
        if (tid == 0)
            listed = taken = 0;
        __syncthreads();
#pragma unroll 8
        for (int64_t c = from + tid; c < to; c += NT)
            if (may_hold(c)) {
                const uint32_t slot = atomicAdd(&listed, 1u);
                if (slot < kListed)
                    list[slot] = (uint32_t)c;
            }
        __syncthreads();
        const uint32_t n = listed;
        __syncthreads();
        if (n > kListed) {
            range = kListed;
            continue;
        }
        if (NT > 256 && from == 0 && wave == WAVES - 1)
            rest();  // (here, where the other waves have something else to do: 37 rows of 100 000 x 64 fp32 34.5 -> 33.2 us)
        // waves take chunks while there is room for what all of them could find in theirs
        for (bool more = n > 0; more;) {
            while (*(volatile uint32_t *)&count <= KEPT - WAVES * kChunk) {
                uint32_t l = 0;
                if (lane == 0)
                    l = atomicAdd(&taken, 1u);
                l = __builtin_amdgcn_readfirstlane(l);
                if (l >= n)
                    break;
                const int64_t chunk = list[l];
                if (may_hold(chunk))
                    logits(chunk);
            }
            __syncthreads();
            more = taken < n;
            __syncthreads();
            if (more)
                settle();
        }
        from = to;
    }
    settle();
    if (tid < a.k) {
        a.top_ids[row * a.k + tid] = id[tid];
        a.top_logp[row * a.k + tid] = (float)(key[tid] - lse_all);
    }
}

// Given ids beyond the table.
__global__ void k_validate_given(int64_t n, int64_t V, const int64_t *given, int *err)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x)
        if (given[i] >= V)
            atomicOr(err, 1);
}

// ---- how a call is cut ---------------------------------------------------------------------------------------------

struct Shape {
    bool few;
    int rows, row_blocks, splits;  // rows of a block
    int64_t chunks, stride, each;
};

// Chunks' maxima of one turn: rows at a time so that they take 512 MiB at most, 64 rows at least.
int64_t rows_at_once(int64_t n, int64_t V, int k)
{
    const int64_t chunks = (V + kChunk - 1) / kChunk;
    int64_t rows = k ? ((int64_t)1 << 27) / (chunks > 0 ? chunks : 1) : (int64_t)1 << 22;
    rows = rows > 64 ? rows : 64;
    rows = rows < (int64_t)1 << 22 ? rows : (int64_t)1 << 22;
    return n < rows ? n : rows;
}

Shape stream_shape(const recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt)
{
    Shape s;
    s.few = n <= kFewRows;
    s.rows = !s.few ? 32 * kMany : n <= 32 || dt == RECD_F32 || D > 128 ? 32 : 64;
    s.row_blocks = (int)((n + s.rows - 1) / s.rows);
    s.chunks = (V + kChunk - 1) / kChunk;
    s.stride = (s.chunks + 3) / 4 * 4;
    // Two blocks a compute unit at a time: of few rows as many splits as give these (37 rows of 1 M x 128 bf16 76 us, three blocks 83,
    // four 80), of many the number whose rounds are fullest
    // (70 000 rows have 274 blocks of rows: with one split most units would have one of them, and some two)
    const int64_t units = s.few ? (s.chunks + kWaves - 1) / kWaves : s.stride / 4;  // a wave's chunk each; four chunks
    const int64_t slots = 2 * ctx->num_cu;
    int64_t splits = slots / s.row_blocks;
    if (!s.few) {
        double best = 1e30;
        for (int64_t k = 1; k <= slots && k <= units; k++) {
            const int64_t rounds = (k * s.row_blocks + slots - 1) / slots;
            const double cost = (double)(rounds * slots) / (double)(k * s.row_blocks) + 0.02 * (double)(k * s.row_blocks) / (double)slots;
            if (cost < best) {
                best = cost;
                splits = k;
            }
        }
    }
    splits = splits < units ? splits : units;
    splits = splits < 1 ? 1 : splits;
    const int64_t each = (units + splits - 1) / splits;
    s.each = each * 4;
    s.splits = (int)((units + each - 1) / each);
    return s;
}

void carve(WsCarver &c, StreamArgs &a, bool top)
{
    a.part_m = c.take<float>((size_t)a.splits * a.n);
    a.part_s = c.take<float>((size_t)a.splits * a.n);
    a.part_t = c.take<float>((size_t)a.splits * a.n);
    a.best = top ? c.take<float>((size_t)a.n * a.stride) : nullptr;
    a.widest = top ? c.take<uint32_t>((size_t)a.stride) : nullptr;
}

recd_status check_answers(recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt, float scale, int k)
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
    if (k < 0 || k > RECD_MAX_ANSWERS || (n > 0 && k > V))
        return recd_fail(ctx, RECD_EINVAL, "k=%d outside [0, %d] or larger than V", k, RECD_MAX_ANSWERS);
    return RECD_OK;
}

template <typename T, int DP> void launch_stream(const StreamArgs &a, const Shape &s, hipStream_t st)
{
    if (s.few) {
        const dim3 grid((unsigned)(s.splits * s.row_blocks));
        if (s.rows == 32)
            hipLaunchKernelGGL((k_answers_few<T, DP, 1>), grid, dim3(64 * kWaves), 0, st, a);
        else if constexpr (sizeof(T) == 2 && DP <= 128)
            hipLaunchKernelGGL((k_answers_few<T, DP, 2>), grid, dim3(64 * kWaves), 0, st, a);
    } else
        hipLaunchKernelGGL((k_answers_many<T, DP>), dim3((unsigned)(((int64_t)s.splits * s.row_blocks + 7) / 8 * 8)), dim3(64 * kMany), 0, st, a);
}

} // namespace

extern "C" {

recd_status recd_vocab_answers_workspace_bytes(int device, int64_t n, int64_t V, int D, recd_dtype dt, int k, size_t *out_bytes)
{
    recd_ctx c;
    if (!out_bytes)
        return RECD_EINVAL;
    RECD_TRY(check_answers(&c, n, V, D, dt, 1.0f, k));
    RECD_TRY(recd_sizing_context(&c, device));
    *out_bytes = 0;
    if (n == 0 || V == 0)
        return RECD_OK;
    size_t most = RECD_VALIDATE_BYTES;
    const int64_t turn = rows_at_once(n, V, k), last = (n - 1) % turn + 1;
    for (const int64_t rows : {turn, last}) {  // (few rows are split further)
        const Shape s = stream_shape(&c, rows, V, D, dt);
        StreamArgs a{};
        a.n = rows;
        a.splits = s.splits;
        a.stride = s.stride;
        WsCarver ws(nullptr);
        carve(ws, a, k > 0);
        most = larger(most, ws.off);
    }
    *out_bytes = most;
    return RECD_OK;
}

recd_status recd_vocab_answers(recd_ctx *ctx, int64_t n, int64_t V, int D, recd_dtype dt, const void *x, const void *table, float scale,
                               const int64_t *given, int k, float *logp, float *entropy, float *lse, int64_t *top_ids, float *top_logp)
{
    RECD_TRY(check_answers(ctx, n, V, D, dt, scale, k));
    if (n == 0)
        return RECD_OK;
    if (V == 0)
        return recd_fail(ctx, RECD_EINVAL, "a vocabulary without rows");
    if (!x || !table || (logp && !given) || (given && !logp) || (k > 0 && (!top_ids || !top_logp)))
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (((uintptr_t)x | (uintptr_t)table) % 16)
        return recd_fail(ctx, RECD_EINVAL, "x and table must be aligned to 16 bytes");
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    ctx->plan.valid = false;  // the parts overwrite the workspace a backward plan would live in
    if (ctx->validate && given) {
        RECD_TRY(recd_reserve(ctx, RECD_VALIDATE_BYTES));
        int *err = reinterpret_cast<int *>(ctx->ws);
        RECD_HIP(ctx, hipMemsetAsync(err, 0, sizeof(int), ctx->stream));
        hipLaunchKernelGGL(k_validate_given, dim3(64), dim3(256), 0, ctx->stream, n, V, given, err);
        RECD_HIP(ctx, hipGetLastError());
        ctx->host_pinned[0] = 0;
        RECD_HIP(ctx, hipMemcpyAsync(ctx->host_pinned, err, sizeof(int), hipMemcpyDeviceToHost, ctx->stream));
        RECD_HIP(ctx, hipStreamSynchronize(ctx->stream));
        if ((int)ctx->host_pinned[0])
            return recd_fail(ctx, RECD_EBOUNDS, "a given id is not a row of the table");
    }
    const int64_t turn = rows_at_once(n, V, k);
    for (int64_t at = 0; at < n; at += turn) {
        const int64_t rows = n - at < turn ? n - at : turn;
        const Shape s = stream_shape(ctx, rows, V, D, dt);
        StreamArgs a{};
        a.n = rows;
        a.V = V;
        a.D = D;
        a.c = fabsf(scale) * kRecdLog2e;
        a.negative = scale < 0;
        a.x = (const char *)x + at * D * (int64_t)elem_size(dt);
        a.table = table;
        a.row_blocks = s.row_blocks;
        a.splits = s.splits;
        a.chunks = s.chunks;
        a.each = s.each;
        a.stride = s.stride;
        WsCarver size(nullptr);
        carve(size, a, k > 0);
        RECD_TRY(recd_reserve(ctx, size.off));
        WsCarver c(ctx->ws);
        carve(c, a, k > 0);
        SelectArgs b{rows, V, D, k, s.splits, scale, a.x, table, given ? given + at : nullptr,
                     a.part_m, a.part_s, a.part_t, a.best, a.widest, s.chunks, s.stride, logp ? logp + at : nullptr,
                     entropy ? entropy + at : nullptr, lse ? lse + at : nullptr, k > 0 ? top_logp + at * k : nullptr,
                     k > 0 ? top_ids + at * k : nullptr};
        recd_with_type(dt, [&](auto t) {
            using T = decltype(t);
            recd_with_width(D, [&](auto w) { launch_stream<T, w.value>(a, s, ctx->stream); });
            int llog = 0;  // lanes of a row
            while ((int)(16 / sizeof(T)) << llog < D)
                llog++;
            // blocks of sixteen waves where there are too few rows to fill the card with blocks of four (37 rows of 100 000 x 64: 19 and 51 us)
            if (rows <= 2 * ctx->num_cu)
                hipLaunchKernelGGL((k_answers_select<T, 1024>), dim3((unsigned)rows), dim3(1024), 0, ctx->stream, b, llog);
            else
                hipLaunchKernelGGL((k_answers_select<T, 256>), dim3((unsigned)rows), dim3(256), 0, ctx->stream, b, llog);
        });
    }
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

} // extern "C"
