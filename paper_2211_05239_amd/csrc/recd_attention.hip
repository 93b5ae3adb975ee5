// Attention inside the lists of jagged rows, and its gradients.
//
// List l has nq query rows and nk key rows; its last query stands at its last key: pos_i = nk - nq + i.
//   z_ij = cap * tanh(scale * q_i . k_j / cap) - slope * |pos_i - j|   (without the tanh where cap = 0)
//   visible: j < lim_i, lim_i = max(pos_i + 1, prefix) with a causal mask, else nk
//   p_ij = exp(z_ij - lse_i) over the visible j, o_i = sum_j p_ij v_j;  a row that sees nothing gives o_i = 0
//   dv_j = sum_i p_ij g_i,  dp_ij = g_i . v_j,  ds_ij = scale * p_ij * (dp_ij - g_i . o_i) * (1 - tanh^2)
//   dq_i = sum_j ds_ij k_j,  dk_j = sum_i ds_ij q_i
//
// The query heads that share a key head are rows of one problem: row r of a (list, key head) is query r / group under
// head r % group of the group.  A tile of one head then reads every key once for the whole group, and the
// gradients by keys and values add the group up in their sums.
//
// Bound by the matrix cores and, beside them, by the vector units: a score costs an exponential (with the cap two and a
// reciprocal, each a quarter of the rate) where it costs 4 d operations of the matrix cores forward.  32 lists of 2048 rows, 8 heads
// on 4 of 128 bf16: 658 us forward (835 TFLOP/s at 4 nq nk d operations; 368 us, 748 under the causal mask) and 2167 us
// backward (634 at 10 nq nk d); 8 heads on 2 of 64 355 us (774) and 1321 (520), with a cap 463 (594) and 1589 (432).  A large
// product reaches 1384; at heads of 128 the vector instructions fill less than half of the time by count, and what the rest of
// the distance goes to is not shown.  Short lists are bound by the chain of one tile (load, two products, exponentials, store) and by what
// is idle in tiles of 32, single rows by the keys' and values' bytes.
//
// Three kernels of one shape: 32 rows of the kept side (queries; in the last kernel keys) a wave in registers, the other
// side streamed through LDS once for scores (by rows) and once for the sums (by columns); the scores never leave
// their lane (recd_mfma.h).  The forward kernel keeps a running maximum and sum.  The backward pass computes the scores
// twice, once for dq and once for dk and dv: 14 nq nk d operations a head instead of 10, and no atomics, so
// the results depend on the sizes alone.
//
// What is rounded to 16 bits for them, beside the operands: the exponentials (as the second product's operand must be) and ds,
// both with an error of half a unit in their last place, which sums average; delta = g . o starts from the output as it was
// stored and is settled to fp32 by the gradients by queries (see there).  Gradients by queries so lie 2.5e-3 (short lists) to 2.9e-3
// from the exact ones (bf16, relative in the 2-norm) where the rounding of the result alone is 1.7e-3.  ds in two roundings would take
// a product more in both kernels (by their count a sixth of the backward pass): not taken.  fp32 rounds nothing.
//
// Tiles of lists are found without a scan: the tiles of list l take the slots from floor(rows before l / R) + l on,
// which never overlap as ceil(n / R) <= floor((before + n) / R) - floor(before / R) + 1.
#include "recd_internal.h"
#include "recd_mfma.h"

#include <math.h>

namespace {

constexpr float kSlack = 8.0f;  // see the running maximum of the forward kernel
template <typename T> constexpr bool kHalf = std::is_same<T, _Float16>::value;
// fp16 exponentials are held 2^7 times larger by the forward pass (at most 2^15 with the slack) and probabilities
// 2^15 times by the backward pass, so that small ones keep their bits (ds: see keep_in_range)
template <typename T> constexpr float kLift = kHalf<T> ? 7.0f : 0.0f;
template <typename T> constexpr float kLiftP = kHalf<T> ? 15.0f : 0.0f;

constexpr int kMostSplits = 1024;  // parts of a tile's keys
constexpr int kMostSorted = 1024;  // lists whose tiles are put in the order of their work

struct Args {
    int G, group, d;              // key heads, query heads of each, elements of a head
    uint32_t by_group;            // ceil(2^32 / group)
    int64_t lists, slots;
    const int2 *tiles;            // {list or -1, tile} of every slot, or null: tiles_per_list slots for every list
    int tiles_per_list, splits;
    int heads;                    // key heads that a block goes through (of one wave; else 1)
    bool last_first;              // without a table: a list's last tiles hold the most work
    const int64_t *q_offsets, *k_offsets;
    const void *q, *k, *v, *out_in, *g;
    int64_t q_stride, k_stride, v_stride, gq_stride, gk_stride, gv_stride;
    float scale, cap;
    const float *slopes;
    const int32_t *prefix;
    int causal;
    void *out, *gq, *gk, *gv;
    float *lse, *delta;           // [q rows][H]
    const float *lse_in;
    float *part_m, *part_l, *part_o;
    int64_t part_rows;            // q rows * H
};

// One list.
struct Problem {
    int64_t q0, k0;
    int nq, nk, rows, pos0, prefix;
    bool causal;

    __device__ inline int query(int row, int group) const { return group == 1 ? row : row / group; }
    // keys [0, limit) are visible to the row; does not fall with the row
    __device__ inline int limit(int row, int group) const { return causal ? limit_at(query(row, group)) : nk; }
    __device__ inline int limit_at(int query) const
    {
        if (!causal)
            return nk;
        const int past = pos0 + query + 1, to = past > prefix ? past : prefix;
        return to < 0 ? 0 : to > nk ? nk : to;
    }
};

// The value of the wave's first lane, which all lanes hold.
__device__ inline int64_t uniform(int64_t v)
{
    return (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}

// The block's tile: false where the slot holds none.  Slots go round the dies; the heads of a slot, whose rows share
// cache lines, follow each other on one die.  Without a table the lists' tiles with the most work come first.
__device__ inline bool find_tile(const Args &a, Problem &p, int &head, int &head_end, int &tile, int &split)
{
    const uint32_t at = blockIdx.x >> 3, turns = a.heads == 1 ? a.G : (a.G + a.heads - 1) / a.heads;
    const uint32_t round = turns == 1 ? at : at / turns;
    const uint32_t unit = round * 8 + (blockIdx.x & 7);
    head = (int)(at - round * turns) * a.heads;
    head_end = head + a.heads < a.G ? head + a.heads : a.G;
    if (unit >= (uint32_t)a.slots * a.splits)
        return false;
    const uint32_t slot = a.splits == 1 ? unit : unit / a.splits;
    split = (int)(unit - slot * a.splits);
    int list;
    if (a.tiles) {
        const int2 t = a.tiles[slot];
        list = __builtin_amdgcn_readfirstlane(t.x);
        tile = __builtin_amdgcn_readfirstlane(t.y);
        if (list < 0)
            return false;
    } else {
        tile = a.tiles_per_list == 1 ? 0 : slot / (uint32_t)a.lists;
        list = slot - tile * (uint32_t)a.lists;
        if (a.last_first)
            tile = a.tiles_per_list - 1 - tile;
    }
    p.q0 = uniform(a.q_offsets[list]);
    p.k0 = uniform(a.k_offsets[list]);
    p.nq = (int)(uniform(a.q_offsets[list + 1]) - p.q0);
    p.nk = (int)(uniform(a.k_offsets[list + 1]) - p.k0);
    p.rows = p.nq * a.group;
    p.pos0 = p.nk - p.nq;
    p.causal = a.causal;
    p.prefix = a.prefix ? __builtin_amdgcn_readfirstlane(a.prefix[list]) : 0;
    return true;
}

// How a block's waves divide a tile: KEPT groups of 32 kept rows, times PHASES that divide the streamed rows and whose
// sums are joined at the end.  With one group every wave streams tiles of its own and waits for nobody; with several, the
// block streams tiles of 32 * PHASES rows that all groups read.
template <typename T, int DP, int KEPT, int PHASES> struct Shape {
    static constexpr bool SHARED = KEPT > 1;
    static constexpr int ROWS = SHARED ? 32 * PHASES : 32, LOADERS = SHARED ? 64 * KEPT * PHASES : 64;
    static constexpr int OWN = SHARED ? 1 : PHASES;  // tiles side by side in LDS
    using Tile = RecdTile<T, ROWS, DP>;
    using Load = RecdStream<T, ROWS, DP, LOADERS>;

    // what the streaming threads wrote is there for the readers
    static __device__ inline void sync()
    {
        if constexpr (SHARED)
            __syncthreads();
        else
            recd_wave_sync();
    }
};

// Adds the phases' sums up into phase 0's, in their order.  pool: 64 * 16 * DT floats for every group.
template <int DT, int PHASES> __device__ inline void join_sums(recd_f32x16 (&o)[DT], float *pool, int group, int phase, int lane)
{
    float *mine = pool + group * (64 * 16 * DT) + lane;
    for (int ph = 1; ph < PHASES; ph++) {
        __syncthreads();
        if (phase == ph)
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    mine[64 * (16 * d + r)] = o[d][r];
        __syncthreads();
        if (phase == 0)
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    o[d][r] += mine[64 * (16 * d + r)];
    }
}

// cap * log2(e) * tanh(x) + (more - base) from x' = 2 log2(e) x, and a quarter of the derivative, (1 - tanh^2) / 4.
// tanh(x) = 1 - 2 r with r = 1 / (1 + e^2x), off by 2^-23 wherever x lies, and the score by 2^-22 of the cap.  That is enough
// beside 16-bit operands for caps up to 256 (6e-5), where the caller's `more` also brings the 1 along (base = cap * log2(e)).
// Elsewhere (WIDE) small x take Lambert's continued fraction, x (945 + 105 x^2 + x^4) / (945 + 420 x^2 + 15 x^4), off by 2e-9 of
// x at 1/2: a score far below its cap keeps all its bits.
enum Cap { NO_CAP, CAP_16, CAP_WIDE };
template <int CAP> struct Capped {
    float cap, cap_n2, base;  // cap * log2(e), -2 times that, and what `more` has to hold besides
    __device__ inline Capped(float c) : cap(c * kRecdLog2e), cap_n2(-2.0f * c * kRecdLog2e), base(CAP == CAP_16 ? c * kRecdLog2e : 0.0f) {}
    __device__ inline float value(float x2, float more, float &quarter) const
    {
        const float r = __builtin_amdgcn_rcpf(1.0f + recd_exp2(x2));
        quarter = r - r * r;
        if constexpr (CAP == CAP_WIDE) {
            const float x = x2 * (0.5f * kRecdLn2), y = x * x;
            float t = 1.0f - 2.0f * r;
            if (fabsf(x) < 0.5f)
                t = x * (945.0f + y * (105.0f + y)) / (945.0f + y * (420.0f + 15.0f * y));
            return cap * t + more;
        }
        return cap_n2 * r + more;
    }
};

template <typename T> __device__ inline void store4(T *p, float a, float b, float c, float d)
{
    T out[4] = {(T)a, (T)b, (T)c, (T)d};
    __builtin_memcpy(p, out, sizeof out);
}

// A head's columns of one row: registers of `sums` are rows of the head's elements.
template <typename T, int DT> __device__ inline void store_columns(T *row, const recd_f32x16 (&o)[DT], float f, int d, int lane)
{
#pragma unroll
    for (int t = 0; t < DT; t++)
        for (int r = 0; r < 16; r += 4) {
            const int col = 32 * t + recd_sums_row(r, lane);
            if (col < d)
                store4<T>(row + col, o[t][r] * f, o[t][r + 1] * f, o[t][r + 2] * f, o[t][r + 3] * f);
        }
}

// o += f * the row's columns.
template <typename T, int DT> __device__ inline void add_columns(recd_f32x16 (&o)[DT], float f, const T *row, int d, int lane)
{
    asm volatile("" : "+v"(lane));  // columns that no register holds through the kernel's loop
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int col = 32 * t + recd_sums_row(r, lane);
            const T *four = row + (col < d ? col : 0);  // (behind the head's end: sums that nobody stores)
            for (int q = 0; q < 4; q++)
                o[t][r + q] += f * (float)four[q];
        }
}

// What is masked enters the products with weight 0, which is not enough where it is an infinity or a NaN: 0 * NaN is a NaN,
// in rows of the tile that do not see it.  Only tiles at the mask's edge hold what some of their rows see and others do not: the
// streamed rows of those are looked through on their way to LDS, zeros take the place of what is not finite there (after the scores,
// which need it as it is), and at the kernel's end every row is given what of it the row does see.  The looking through costs
// an operation a word of such tiles, and what is found the reading of those tiles' rows once more, however much it is: 2048 rows, 4
// heads on 2 of 128 bf16, both passes 147 us, with one infinite gradient 191, with nothing else 253, with one infinite value 168.

// Whether any of a block's waves says so, or a wave that streams for itself.
template <bool SHARED, int WAVES> __device__ inline bool any_wave(bool mine, int (&says)[WAVES], int wave, int lane)
{
    if constexpr (SHARED) {
        if (lane == 0)
            says[wave] = mine;
        __syncthreads();
        int any = 0;
        for (int w = 0; w < WAVES; w++)
            any |= says[w];
        return __builtin_amdgcn_readfirstlane(any) != 0;
    }
    return mine;
}

// Adds what is not finite in the streamed rows [s0, s1) to the sums of the lanes whose column sees it: itself under weights that
// are positive, else a NaN.
template <bool POSITIVE, typename T, int DT, typename Row, typename Sees>
__device__ inline void add_not_finite(int s0, int s1, int d, Row row_of, Sees sees, recd_f32x16 (&o)[DT], int lane)
{
    asm volatile("" : "+v"(lane));  // columns that no register holds through the kernel's loop
#pragma unroll 1
    for (int s = s0; s < s1; s++) {
        if (!sees(s))
            continue;
        const T *row = row_of(s);
#pragma unroll
        for (int t = 0; t < DT; t++)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int col = 32 * t + recd_sums_row(r, lane);
                const T *four = row + (col < d ? col : 0);  // (behind the head's end: sums that nobody stores)
                for (int q = 0; q < 4; q++) {
                    const float x = (float)four[q];
                    o[t][r + q] += POSITIVE ? (fabsf(x) < INFINITY ? 0.0f : x) : x - x;
                }
            }
    }
}

// Waves that a SIMD is to hold at once, as far as the registers go round: two hide each other's waits and fill the
// matrix cores and the vector units in turn.
template <typename T, int DP, int KEPT> constexpr int kResident = (sizeof(T) == 4 && DP > 32) || (KEPT == 1 && DP > 64) ? 1 : 2;

// The gradients by queries of 64 wide heads, whose registers pass a third of all by a few: three with what does not fit in memory, in
// place of two.  32 lists of 2048 rows, 8 heads on 2, with a cap, backward 1566 us against 1654.
template <typename T, int DP, int KEPT> constexpr int kResidentQ = sizeof(T) == 2 && DP == 64 && KEPT > 1 ? 3 : kResident<T, DP, KEPT>;

// 32 query rows a wave.  The loop is pipelined over tiles of 32 keys: one turn multiplies the next tile's scores and the
// current one's sums while the current scores become exponentials.  The caps, biases and masks of the next scores, and
// the check of the running maximum, stand behind it.  Three buffers in LDS make it one barrier a turn; waves that stream for
// themselves need two and none.
template <typename T, int DP, int KEPT, int PHASES, int CAP>
__global__ __launch_bounds__(64 * KEPT * PHASES, (kResident<T, DP, KEPT>)) void k_attention(Args a)
{
    using S = Shape<T, DP, KEPT, PHASES>;
    static_assert(KEPT == 1 || PHASES == 1);
    constexpr int KS = DP / 16, DT = DP / 32, BUFS = S::SHARED ? 3 : 2;
    using Mma = RecdMma<T>;
    using Frag = typename Mma::Frag;
    __shared__ struct {
        typename S::Tile k[S::OWN][BUFS], v[S::OWN][BUFS];
    } lds;
    __shared__ int says[KEPT * PHASES];
    Problem p;
    int head, tile, split;
    int head_end;
    if (!find_tile(a, p, head, head_end, tile, split))
        return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kept = wave % KEPT, phase = wave / KEPT;
    const int tid = S::SHARED ? threadIdx.x : lane;
    typename S::Tile *const kt = lds.k[S::SHARED ? 0 : phase], *const vt = lds.v[S::SHARED ? 0 : phase];
    const int first = tile * 32 * KEPT, end = first + 32 * KEPT < p.rows ? first + 32 * KEPT : p.rows;  // the block's rows
    if (first >= end)
        return;
    const int row0 = first + 32 * kept, row = row0 + (lane & 31);
    const bool there = row < p.rows;
    const int query = p.query(row, a.group), head_in = row - query * a.group;
    const int lim = there ? p.limit(row, a.group) : 0;
    const int wave_last = row0 + 31 < p.rows ? row0 + 31 : p.rows - 1;
    const int wave_end = row0 < p.rows ? p.limit(wave_last, a.group) : 0;
    const int wave_full = row0 + 32 <= p.rows ? p.limit(row0, a.group) : 0;  // keys that every row sees
    const int tiles = (p.limit(end - 1, a.group) + 31) / 32;
    const int edge = p.limit(first, a.group) / 32;  // the block's first tile that not all of its rows see
    const int part = split * PHASES + phase, parts = a.splits * PHASES;
    const int each = parts == 1 ? tiles : (tiles + parts - 1) / parts;  // tiles of a part
    const int t0 = part * each < tiles ? part * each : tiles, t1 = t0 + each < tiles ? t0 + each : tiles;
    const int wave_t1 = (wave_end + 31) / 32 < t1 ? (wave_end + 31) / 32 : t1;
    const int H = a.G * a.group;
    const int64_t q_row = p.q0 + query, at_row = q_row * H + head * a.group + head_in;
    const float slope = a.slopes && there ? a.slopes[head * a.group + head_in] * kRecdLog2e : 0.0f;
    const int pos = p.pos0 + query;
    // the sign of the scale goes into the queries; what is neither capped nor biased stays unscaled until the exponent
    const float scale = fabsf(a.scale), c = scale * kRecdLog2e;
    const bool plain = !CAP && !a.slopes && c > 0.0f;
    const float by = plain ? c : 1.0f;
    const Capped<CAP> capped(a.cap);
    const float to_cap = CAP ? 2.0f * kRecdLog2e * scale / a.cap : 0.0f;

    Frag qf[KS];
#pragma unroll
    for (int k = 0; k < KS; k++) {
        qf[k] = recd_row_frag<T>((const T *)a.q + q_row * a.q_stride + (int64_t)(head * a.group + head_in) * a.d, 16 * k, a.d, there,
                                 lane);
        if (a.scale < 0.0f)
            qf[k] = recd_negated(qf[k]);
    }
    float m = -INFINITY, l = 0.0f;
    recd_f32x16 o[DT], s[2];
#pragma unroll
    for (int d = 0; d < DT; d++)
        o[d] = recd_f32x16{};
    typename S::Load ks, vs;
    if (a.d < DP)
        for (int b = 0; b < BUFS; b++) {
            ks.clear_behind(tid, kt[b], a.d);
            vs.clear_behind(tid, vt[b], a.d);
        }
    auto load = [&](int t) {
        const int64_t at = p.k0 + t * 32;
        ks.load_rows(tid, (const T *)a.k + at * a.k_stride + head * a.d, p.nk - t * 32, a.d, (uint32_t)a.k_stride * sizeof(T));
        vs.load_rows(tid, (const T *)a.v + at * a.v_stride + head * a.d, p.nk - t * 32, a.d, (uint32_t)a.v_stride * sizeof(T));
    };
    auto scores = [&](const typename S::Tile &keys, recd_f32x16 &x) {
        x = recd_f32x16{};
#pragma unroll
        for (int k = 0; k < KS; k++)
            x = Mma::mul(keys.rows(0, 16 * k, lane), qf[k], x);
    };
    auto settle = [&](int j0, recd_f32x16 &x) {
        if (a.slopes) {
            const float far = (float)(pos - j0 - (lane >> 5));  // (whole numbers: positions may pass 2^24)
#pragma unroll
            for (int r = 0; r < 16; r++) {
                const float bias = capped.base - slope * fabsf(far - (float)recd_score_row(r, 0));
                float unused;
                x[r] = CAP ? capped.value(x[r] * to_cap, bias, unused) : x[r] * c + bias;
            }
        } else if (!plain) {
#pragma unroll
            for (int r = 0; r < 16; r++) {
                float unused;
                x[r] = CAP ? capped.value(x[r] * to_cap, capped.base, unused) : x[r] * c;
            }
        }
        if (j0 + 32 > wave_full) {
            asm volatile("");  // a branch: only the tiles at the mask's edge pay for it
#pragma unroll
            for (int r = 0; r < 16; r++)
                x[r] = j0 + recd_score_row(r, lane) >= lim ? -INFINITY : x[r];
        }
        float top = x[0];
#pragma unroll
        for (int r = 1; r < 16; r++)
            top = fmaxf(top, x[r]);
        top = fmaxf(top, __shfl_xor(top, 32)) * by - kLift<T>;
        // the maximum moves only where it grows by more than 2^kSlack: the sums are rarely rescaled
        if (__any(top > m + kSlack)) {
            const float now = fmaxf(m, top);
            const float f = now == m ? 1.0f : recd_exp2(m - now);
            m = now;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    o[d][r] *= f;
        }
    };
    bool odd = false;  // the wave's threads have seen what is not finite at the edge
    auto store = [&](int t, int b) {
        ks.store(tid, kt[b], a.d);
        vs.store(tid, vt[b], a.d);
        if (t >= edge && __any(vs.not_finite(tid))) {
            vt[b].make_finite(tid, S::LOADERS);  // (what the thread has stored itself)
            odd = true;
        }
    };
    if (t0 < t1) {
        load(t0);
        store(t0, 0);
        if (t0 + 1 < t1)
            load(t0 + 1);
        S::sync();
        if (t0 < wave_t1) {
            scores(kt[0], s[0]);
            settle(t0 * 32, s[0]);
        }
    }
    int buf = 0;
    auto turn = [&](int t, recd_f32x16 &now, recd_f32x16 &then) {
        const int next = buf + 1 == BUFS ? 0 : buf + 1;
        if (t + 1 < t1) {
            store(t + 1, next);
            if (t + 2 < t1)
                load(t + 2);
        }
        S::sync();
        if (t < wave_t1) {
            scores(kt[next], then);  // (behind the wave's last tile: of what lies there, for nobody)
            const float from = m == -INFINITY ? 0.0f : m;  // a row that has seen nothing yet
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; r++) {
                now[r] = recd_exp2(now[r] * by - from);
                sum += now[r];
            }
            l += sum;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const Frag pf = recd_sums_frag<T>(now, h);
#pragma unroll
                for (int d = 0; d < DT; d++)
                    o[d] = Mma::mul(vt[buf].columns(16 * h, 32 * d, lane), pf, o[d]);
            }
            if (t + 1 < wave_t1)
                settle((t + 1) * 32, then);
        }
        buf = next;
    };
    for (int t = t0; t < t1; t += 2) {
        turn(t, s[0], s[1]);
        if (t + 1 < t1)
            turn(t + 1, s[1], s[0]);
    }
    if (t1 > edge && any_wave<S::SHARED>(odd, says, wave, lane)) {
        const T *values = (const T *)a.v + p.k0 * a.v_stride + head * a.d;
        add_not_finite<true, T>(t0 > edge ? t0 * 32 : edge * 32, t1 * 32 < p.nk ? t1 * 32 : p.nk, a.d,
                                [&](int j) { return values + j * a.v_stride; }, [&](int j) { return j < lim; }, o, lane);
    }
    l += __shfl_xor(l, 32);
    if constexpr (PHASES > 1) {  // in the order of the phases: the larger maximum, both sums scaled to it
        float *const pool = reinterpret_cast<float *>(&lds);
        static_assert(sizeof(lds) >= 64 * (16 * DT + 2) * sizeof(float));
        for (int ph = 1; ph < PHASES; ph++) {
            __syncthreads();
            if (phase == ph) {
                pool[lane] = m;
                pool[64 + lane] = l;
#pragma unroll
                for (int d = 0; d < DT; d++)
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        pool[64 * (2 + 16 * d + r) + lane] = o[d][r];
            }
            __syncthreads();
            if (phase == 0) {
                const float other = pool[lane], top = fmaxf(m, other), from = top == -INFINITY ? 0.0f : top;
                const float f = recd_exp2(m - from), g = recd_exp2(other - from);
                m = top;
                l = l * f + pool[64 + lane] * g;
#pragma unroll
                for (int d = 0; d < DT; d++)
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        o[d][r] = o[d][r] * f + pool[64 * (2 + 16 * d + r) + lane] * g;
            }
        }
    }
    if (phase)
        return;
    if (!there)
        return;
    if (a.splits > 1) {
        const int64_t at = split * a.part_rows + at_row;
        if (lane < 32) {
            a.part_m[at] = m;
            a.part_l[at] = l;
        }
        store_columns<float, DT>(a.part_o + at * a.d, o, 1.0f, a.d, lane);
    } else {
        if (a.lse && lane < 32)
            a.lse[at_row] = (m + log2f(l)) * kRecdLn2;  // -inf where l = 0
        store_columns<T, DT>((T *)a.out + at_row * a.d, o, l == 0.0f ? 0.0f : 1.0f / l, a.d, lane);
    }
}

// The forward kernel for lists of few rows: a wave to itself goes through one head after the other, whose rows are on
// their way while it works at the one before, so that a wave finds its list once for all of them.
template <typename T, int DP, int CAP> __global__ __launch_bounds__(64, (sizeof(T) == 2 && DP <= 32 ? 4 : kResident<T, DP, 1>)) void k_attention_one(Args a)
{
    constexpr int KS = DP / 16, DT = DP / 32;
    using Mma = RecdMma<T>;
    using Frag = typename Mma::Frag;
    using S = Shape<T, DP, 1, 1>;
    __shared__ typename S::Tile kt, vt;
    Problem p;
    int head, head_end, tile, split;
    if (!find_tile(a, p, head, head_end, tile, split))
        return;
    const int lane = threadIdx.x, row0 = tile * 32, row = row0 + (lane & 31);
    if (row0 >= p.rows)
        return;
    const bool there = row < p.rows;
    const int query = p.query(row, a.group), head_in = row - query * a.group;
    const int lim = there ? p.limit(row, a.group) : 0;
    const int full = row0 + 32 <= p.rows ? p.limit(row0, a.group) : 0;
    const int end = p.limit(row0 + 31 < p.rows ? row0 + 31 : p.rows - 1, a.group), tiles = (end + 31) / 32;
    const int each = a.splits == 1 ? tiles : (tiles + a.splits - 1) / a.splits;  // tiles of a split
    const int t0 = split * each < tiles ? split * each : tiles, t1 = t0 + each < tiles ? t0 + each : tiles;
    const int H = a.G * a.group;
    const int64_t q_row = p.q0 + query;
    const int pos = p.pos0 + query;
    const float c = a.scale * kRecdLog2e;
    const Capped<CAP> capped(a.cap);
    const float to_cap = CAP ? 2.0f * kRecdLog2e * a.scale / a.cap : 0.0f;
    Frag qf[KS], qn[KS];
    float slope = 0.0f, slope_n = 0.0f, m = -INFINITY, l = 0.0f;
    recd_f32x16 o[DT];
    typename S::Load ks, vs;
    if (a.d < DP) {
        ks.clear_behind(lane, kt, a.d);
        vs.clear_behind(lane, vt, a.d);
    }
    auto load_q = [&](int hd) {
        const int h = hd * a.group + head_in;
#pragma unroll
        for (int k = 0; k < KS; k++)
            qn[k] = recd_row_frag<T>((const T *)a.q + q_row * a.q_stride + (int64_t)h * a.d, 16 * k, a.d, there, lane);
        slope_n = a.slopes && there ? a.slopes[h] * kRecdLog2e : 0.0f;
    };
    auto load = [&](int hd, int t) {
        const int64_t at = p.k0 + t * 32;
        ks.load_rows(lane, (const T *)a.k + at * a.k_stride + hd * a.d, p.nk - t * 32, a.d, (uint32_t)a.k_stride * sizeof(T));
        vs.load_rows(lane, (const T *)a.v + at * a.v_stride + hd * a.d, p.nk - t * 32, a.d, (uint32_t)a.v_stride * sizeof(T));
    };
    bool odd = false;  // something that is not finite in the head's tiles (few, and most of them at the mask's edge)
    auto take = [&]() {
        odd = false;
        slope = slope_n;
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; k++)
            qf[k] = qn[k];
#pragma unroll
        for (int d = 0; d < DT; d++)
            o[d] = recd_f32x16{};
    };
    auto write = [&]() {
        const float sum = l + __shfl_xor(l, 32);
        const int64_t at_row = q_row * H + head * a.group + head_in;
        if (!there)
            return;
        if (a.splits > 1) {
            const int64_t at = split * a.part_rows + at_row;
            if (lane < 32) {
                a.part_m[at] = m;
                a.part_l[at] = sum;
            }
            store_columns<float, DT>(a.part_o + at * a.d, o, 1.0f, a.d, lane);
            return;
        }
        if (a.lse && lane < 32)
            a.lse[at_row] = (m + log2f(sum)) * kRecdLn2;  // -inf where the sum is 0
        store_columns<T, DT>((T *)a.out + at_row * a.d, o, sum == 0.0f ? 0.0f : 1.0f / sum, a.d, lane);
    };
    load_q(head);
    if (t0 < t1)
        load(head, t0);
    take();
    if (t0 == t1)
        for (; head < head_end; head++)  // no keys
            write();
    for (int t = t0; t < t1;) {
        S::sync();
        ks.store(lane, kt, a.d);
        vs.store(lane, vt, a.d);
        const bool clear = __any(vs.not_finite(lane));
        S::sync();
        const bool last = t + 1 == t1, more = last && head + 1 < head_end;
        if (!last || more)
            load(more ? head + 1 : head, more ? t0 : t + 1);
        if (more)
            load_q(head + 1);
        const int j0 = t * 32;
        recd_f32x16 s = {};
#pragma unroll
        for (int k = 0; k < KS; k++)
            s = Mma::mul(kt.rows(0, 16 * k, lane), qf[k], s);
        if (clear) {
            vt.make_finite(lane, 64);
            S::sync();
            odd = true;
        }
        auto finish = [&](auto registers) {
            constexpr int NR = registers.value;
            if (a.slopes) {
                const float far = (float)(pos - j0 - (lane >> 5));  // (whole numbers: positions may pass 2^24)
#pragma unroll
                for (int r = 0; r < NR; r++) {
                    const float bias = capped.base - slope * fabsf(far - (float)recd_score_row(r, 0));
                    float unused;
                    s[r] = CAP ? capped.value(s[r] * to_cap, bias, unused) : s[r] * c + bias;
                }
            } else {
#pragma unroll
                for (int r = 0; r < NR; r++) {
                    float unused;
                    s[r] = CAP ? capped.value(s[r] * to_cap, capped.base, unused) : s[r] * c;
                }
            }
            if (j0 + 2 * NR > full) {
                asm volatile("");
                const int to = lim - j0 - (lane >> 5);
#pragma unroll
                for (int r = 0; r < NR; r++)
                    s[r] = recd_score_row(r, 0) >= to ? -INFINITY : s[r];
            }
            float top = s[0];
#pragma unroll
            for (int r = 1; r < NR; r++)
                top = fmaxf(top, s[r]);
            top = fmaxf(top, __shfl_xor(top, 32)) - kLift<T>;
            const float now = fmaxf(m, top), from = now == -INFINITY ? 0.0f : now;
            if (t > t0) {
                const float f = recd_exp2(m - from);
                l *= f;
#pragma unroll
                for (int d = 0; d < DT; d++)
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        o[d][r] *= f;
            }
            m = now;
#pragma unroll
            for (int r = 0; r < NR; r++) {
                s[r] = recd_exp2(s[r] - from);
                l += s[r];
            }
#pragma unroll
            for (int h = 0; h < NR / 8; h++) {
                const Frag pf = recd_sums_frag<T>(s, h);
#pragma unroll
                for (int d = 0; d < DT; d++)
                    o[d] = Mma::mul(vt.columns(16 * h, 32 * d, lane), pf, o[d]);
            }
        };
        if (end - j0 <= 16)  // the other registers hold no key of the list
            finish(std::integral_constant<int, 8>{});
        else
            finish(std::integral_constant<int, 16>{});
        t++;
        if (last) {
            if (odd) {
                const T *values = (const T *)a.v + p.k0 * a.v_stride + head * a.d;
                add_not_finite<true, T>(t0 * 32, t1 * 32 < p.nk ? t1 * 32 : p.nk, a.d, [&](int j) { return values + j * a.v_stride; },
                                        [&](int j) { return j < lim; }, o, lane);
            }
            write();
        }
        if (more) {
            head++;
            t = t0;
            take();
        }
    }
}

// Joins the splits of the forward pass where they are few: 2^dlog threads a row, four elements each.
template <typename T>
__global__ __launch_bounds__(256) void k_attention_join(int64_t rows, int d, int dlog, int splits,
                                                        const float *__restrict__ part_m, const float *__restrict__ part_l,
                                                        const float *__restrict__ part_o, T *out, float *lse)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i >> dlog;
    const int col = (int)(i & ((1 << dlog) - 1)) * 4;
    if (row >= rows || col >= d)
        return;
    float m = -INFINITY;
    for (int s = 0; s < splits; s++)
        m = fmaxf(m, part_m[s * rows + row]);
    const float from = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    recd_f32x4 o = {};
    for (int s = 0; s < splits; s++) {
        const float f = recd_exp2(part_m[s * rows + row] - from);
        l += f * part_l[s * rows + row];
        const recd_f32x4 x = *reinterpret_cast<const recd_f32x4 *>(part_o + (s * rows + row) * d + col);
        for (int e = 0; e < 4; e++)
            o[e] += f * x[e];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    store4<T>(out + row * d + col, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (lse && col == 0)
        lse[row] = (m + log2f(l)) * kRecdLn2;
}

// The same for many splits: a block a row, the splits dealt to its threads (one thread to a split for the
// weights, 2^dlog threads with four elements each for the sums), so that no chain of loads is as long as the splits are
// many.  A whole call with it and with the other, one query of 8 heads of 64 fp16 against 30 000 keys (58 splits) 14 and 30 us,
// against 200 000 (256 splits) 29 and 113.
template <typename T>
__global__ __launch_bounds__(256) void k_attention_join_many(int64_t rows, int d, int dlog, int splits,
                                                             const float *__restrict__ part_m, const float *__restrict__ part_l,
                                                             const float *__restrict__ part_o, T *out, float *lse)
{
    __shared__ float f[kMostSplits], wave_m[4], wave_l[4];
    __shared__ recd_f32x4 sums[256];
    const int tid = threadIdx.x, wave = tid >> 6;
    const int64_t row = blockIdx.x;
    float m = -INFINITY;
    for (int s = tid; s < splits; s += 256) {
        f[s] = part_m[s * rows + row];
        m = fmaxf(m, f[s]);
    }
    for (int o = 32; o; o >>= 1)
        m = fmaxf(m, __shfl_xor(m, o));
    if ((tid & 63) == 0)
        wave_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3]));
    const float from = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    for (int s = tid; s < splits; s += 256) {
        f[s] = recd_exp2(f[s] - from);
        l += f[s] * part_l[s * rows + row];
    }
    for (int o = 32; o; o >>= 1)
        l += __shfl_xor(l, o);
    if ((tid & 63) == 0)
        wave_l[wave] = l;
    __syncthreads();
    l = wave_l[0] + wave_l[1] + wave_l[2] + wave_l[3];
    const int col = (tid & ((1 << dlog) - 1)) * 4, lot = tid >> dlog, lots = 256 >> dlog;
    recd_f32x4 o = {};
    if (col < d)
        for (int s0 = lot; s0 < splits; s0 += 4 * lots) {
            recd_f32x4 x[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int s = s0 + i * lots < splits ? s0 + i * lots : s0;
                x[i] = *reinterpret_cast<const recd_f32x4 *>(part_o + (s * rows + row) * d + col);
            }
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (s0 + i * lots < splits)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        o[e] += f[s0 + i * lots] * x[i][e];
        }
    sums[tid] = o;
    __syncthreads();
    if (lot || col >= d)
        return;
    for (int i = 1; i < lots; i++)
#pragma unroll
        for (int e = 0; e < 4; e++)
            o[e] += sums[(i << dlog) + tid][e];
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    store4<T>(out + row * d + col, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (lse && tid == 0)
        lse[row] = (m + log2f(l)) * kRecdLn2;
}

// A side whose tiles are listed.  `keys`: its tiles are of keys, else of queries, `group` rows each.
struct Side {
    int64_t slots;
    int group, R;
    bool keys;
    int2 *tiles;
};

// {list, tile} of a side's slots; a row of blocks for each side.
__global__ __launch_bounds__(256) void k_attention_tiles(int64_t lists, const int64_t *__restrict__ q_offsets,
                                                         const int64_t *__restrict__ k_offsets, Side one, Side two)
{
    const Side &side = blockIdx.y ? two : one;
    const int64_t *offsets = side.keys ? k_offsets : q_offsets;
    const int64_t list = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (list >= lists)
        return;
    const int64_t b = offsets[list] * side.group, e = offsets[list + 1] * side.group;
    const int64_t s0 = b / side.R + list, n = (e - b + side.R - 1) / side.R;
    const int64_t s1 = list + 1 < lists ? e / side.R + list + 1 : side.slots;
    for (int64_t s = s0 < 0 ? 0 : s0; s < s1 && s < side.slots; s++)
        side.tiles[s] = s - s0 < n ? make_int2((int)list, (int)(s - s0)) : make_int2(-1, 0);
}

// The same for few lists (a block for each side), in the order of the tiles' work, most first: lists of a few very
// different lengths would otherwise leave most compute units to wait for the last long one: in the order of the lists against
// this, 8 lists of up to 4096 rows forward and backward 1006 / 725 us, 24 of up to 2048 forward 182 / 157, 61 of up to 500 161 /
// 137; single rows of 8 lists lose 5 us of 25 to the sorting block.  Tiles of about equal work stand in any order.
__global__ __launch_bounds__(1024) void k_attention_tiles_by_work(int lists, bool causal, const int64_t *__restrict__ q_offsets,
                                                                  const int64_t *__restrict__ k_offsets,
                                                                  const int32_t *__restrict__ prefix, Side one, Side two)
{
    __shared__ int nq[kMostSorted], nk[kMostSorted], pre[kMostSorted], count[256], wave_sum[4], most;
    const Side &side = blockIdx.x ? two : one;
    const int group = side.group, R = side.R;
    if (threadIdx.x < 256)
        count[threadIdx.x] = 0;
    if (threadIdx.x == 0)
        most = 1;
    __syncthreads();
    int top = 1;
    for (int l = threadIdx.x; l < lists; l += 1024) {
        nq[l] = (int)(q_offsets[l + 1] - q_offsets[l]);
        nk[l] = (int)(k_offsets[l + 1] - k_offsets[l]);
        pre[l] = prefix ? prefix[l] : 0;
        const int n = side.keys ? nq[l] : nk[l];
        top = n > top ? n : top;
    }
    atomicMax(&most, top);
    __syncthreads();
    // rows (of queries or keys) that tile i of list l goes through, in 256ths of the longest list's
    const float unit = 255.0f / (float)most;
    auto bucket = [&](int l, int i) {
        int work;
        if (side.keys) {
            const int first = i * R, pos0 = nk[l] - nq[l];
            work = causal && pre[l] <= first && first > pos0 ? nq[l] - (first - pos0) : nq[l];
        } else {
            int last = group == 1 ? (i + 1) * R : (int)((int64_t)(i + 1) * R / group);
            last = last < nq[l] ? last : nq[l];
            int end = nk[l] - nq[l] + last;
            end = end > pre[l] ? end : pre[l];
            work = causal && end < nk[l] ? end : nk[l];
        }
        const int b = 255 - (int)((float)(work < 0 ? 0 : work) * unit);
        return b < 0 ? 0 : b;
    };
    const int lane = threadIdx.x & 31;
    for (int l = threadIdx.x >> 5; l < lists; l += 32) {
        const int n = ((side.keys ? nk[l] : nq[l] * group) + R - 1) / R;
        for (int i = lane; i < n; i += 32)
            atomicAdd(&count[bucket(l, i)], 1);
    }
    __syncthreads();
    // where every bucket starts
    int mine = 0, sum = 0;
    if (threadIdx.x < 256) {
        sum = mine = count[threadIdx.x];
        for (int o = 1; o < 64; o <<= 1) {
            const int other = __shfl_up(sum, o);
            sum += (int)(threadIdx.x & 63) >= o ? other : 0;
        }
        if ((threadIdx.x & 63) == 63)
            wave_sum[threadIdx.x >> 6] = sum;
    }
    __syncthreads();
    if (threadIdx.x < 256) {
        for (int w = 0; w < (int)(threadIdx.x >> 6); w++)
            sum += wave_sum[w];
        count[threadIdx.x] = sum - mine;
    }
    const int total = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    __syncthreads();
    for (int l = threadIdx.x >> 5; l < lists; l += 32) {
        const int n = ((side.keys ? nk[l] : nq[l] * group) + R - 1) / R;
        for (int i = lane; i < n; i += 32) {
            const int at = atomicAdd(&count[bucket(l, i)], 1);
            if (at < side.slots)
                side.tiles[at] = make_int2(l, i);
        }
    }
    for (int64_t s = total + threadIdx.x; s < side.slots; s += 1024)
        side.tiles[s] = make_int2(-1, 0);
}

// fp16 holds ds larger by a power of two of every column's own (a query's, a key's), which falls where a tile's largest
// leaves the range: to between 2^10 and 2^11, so that few tiles pass 2^15 again.  Terms down to 2^-24 of a column's largest so keep
// all their bits, whatever other rows, heads and lists hold.  Gives the factor by which x and the sums o have become smaller.
constexpr float kFirstLift = 0x1p60f;  // products of two fp16 heads are less than 2^40
template <int NR, int DT> __device__ inline float keep_in_range(recd_f32x16 &x, recd_f32x16 (&o)[DT])
{
    float top = fabsf(x[0]);
#pragma unroll
    for (int r = 1; r < NR; r++)
        top = fmaxf(top, fabsf(x[r]));
    top = fmaxf(top, __shfl_xor(top, 32));
    const bool leaves = top > 0x1p15f && top < INFINITY;
    if (!__any(leaves))
        return 1.0f;
    const float f = leaves ? __uint_as_float((264u << 23) - (__float_as_uint(top) & 0x7f800000u)) : 1.0f;
#pragma unroll
    for (int r = 0; r < NR; r++)
        x[r] *= f;
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
        for (int r = 0; r < 16; r++)
            o[t][r] *= f;
    return f;
}

// 1 / a power of two
__device__ inline float inverse_power(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }

template <int DT> __device__ inline void scale_sums(recd_f32x16 (&o)[DT], float f)
{
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
        for (int r = 0; r < 16; r++)
            o[t][r] *= f;
}

// 32 query rows a wave, keys and values stream past.
//
// With 16 bits delta has to settle.  ds_j = p_j (dp_j - delta) is the difference of two nearly equal numbers where one key has almost
// all of a row's weight, and delta = g . o of the output as it was rounded is off by e, up to half a unit of its last place: at
// p = 0.95 .. 0.99 that alone is 7 % of the row's gradient in the median and more than all of it at worst (bf16, by calculation in 64
// bits with the output rounded), at 0.99 .. 0.999 85 %.
// As the p_j sum up to 1, the sum of p_j (dp_j - delta) is -e, and the gradients by keys take delta without it.  A row's own
// gradient needs sum_j p_j k_j for that, another product; taking the keys from the heaviest one's place, sum_j ds_j (k_j - k*),
// leaves e (sum_j p_j k_j - k*), which vanishes as the weight on one key (or on several that are the same) grows, where e
// counts; elsewhere ds is large beside it.  Where a wave has all of a list's keys at once, e is known before ds is made.  Measured, one
// list of 700 rows: bf16 0.2 to 0.35 % in the median for all p and 4 % in the worst row, fp16 0.03 to 0.05 % with worst rows below
// 0.5 %, but at p > 0.999 2 % (heads of 64) and 12 % (128).  fp32 has delta to 2^-24 already.
// (that product added instead: backward 4 to 12 % slower at heads of 64, 10 to 30 in lists of one wave, 22 to 35, with spills, at heads
// of 128; the rows in question done again: 10 to 15 % on long lists with slopes.)
// It costs an addition, half a maximum and in few tiles a search a score, and registers: short lists of 32 wide heads hold three waves
// a SIMD where they held four, and their gradients by queries take 66 us for 50 (that the waves are the cause is not shown).
template <typename T, int DP, int KEPT, int PHASES, int CAP>
__global__ __launch_bounds__(64 * KEPT * PHASES, (kResidentQ<T, DP, KEPT>)) void k_attention_grad_q(Args a)
{
    using S = Shape<T, DP, KEPT, PHASES>;
    static_assert(KEPT == 1 || PHASES == 1);
    constexpr bool ONE = KEPT * PHASES == 1, SETTLES = sizeof(T) == 2;
    constexpr int KS = DP / 16, DT = DP / 32, BUFS = S::SHARED ? 2 : 1;
    using Mma = RecdMma<T>;
    using Frag = typename Mma::Frag;
    __shared__ struct {
        typename S::Tile k[S::OWN][BUFS], v[S::OWN][BUFS];
    } lds;
    __shared__ int says[2][KEPT * PHASES];
    __shared__ float of_phase[SETTLES && PHASES > 1 ? PHASES : 1][4][64];
    Problem p;
    int head, head_end, tile, split;
    if (!find_tile(a, p, head, head_end, tile, split))
        return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kept = wave % KEPT, phase = wave / KEPT;
    const int tid = S::SHARED ? threadIdx.x : lane;
    typename S::Tile *const kt = lds.k[S::SHARED ? 0 : phase], *const vt = lds.v[S::SHARED ? 0 : phase];
    const int first = tile * 32 * KEPT, end = first + 32 * KEPT < p.rows ? first + 32 * KEPT : p.rows;
    if (first >= end)
        return;
    const int row0 = first + 32 * kept, row = row0 + (lane & 31);
    const bool there = row < p.rows;
    const int query = p.query(row, a.group), head_in = row - query * a.group;
    const int lim = there ? p.limit(row, a.group) : 0;
    const int wave_last = row0 + 31 < p.rows ? row0 + 31 : p.rows - 1;
    const int wave_end = row0 < p.rows ? p.limit(wave_last, a.group) : 0;
    const int wave_full = row0 + 32 <= p.rows ? p.limit(row0, a.group) : 0;
    const int tiles = (p.limit(end - 1, a.group) + 31) / 32, t0 = tiles * phase / PHASES, t1 = tiles * (phase + 1) / PHASES;
    // the block's first tile that not all of its rows see (a wave that has few tiles looks all of them through)
    const int edge = ONE ? 0 : p.limit(first, a.group) / 32;
    const int H = a.G * a.group;
    const int64_t q_row = p.q0 + query;
    const int pos = p.pos0 + query;
    float lift = kHalf<T> ? kFirstLift : 1.0f;
    const float c = a.scale * kRecdLog2e;
    const Capped<CAP> capped(a.cap);
    const float to_cap = CAP ? 2.0f * kRecdLog2e * a.scale / a.cap : 0.0f;

    // delta = g . o, to begin with of the output as it is stored
    const int h = head * a.group + head_in;
    const int64_t at_row = q_row * H + h;
    Frag qf[KS], gf[KS];
    float delta = 0.0f;
#pragma unroll
    for (int k = 0; k < KS; k++) {
        qf[k] = recd_row_frag<T>((const T *)a.q + q_row * a.q_stride + (int64_t)h * a.d, 16 * k, a.d, there, lane);
        gf[k] = recd_row_frag<T>((const T *)a.g + at_row * a.d, 16 * k, a.d, there, lane);
        const Frag out = recd_row_frag<T>((const T *)a.out_in + at_row * a.d, 16 * k, a.d, there, lane);
#pragma unroll
        for (int e = 0; e < 8; e++)
            delta += (float)gf[k][e] * (float)out[e];
    }
    delta += __shfl_xor(delta, 32);
    const float stored = delta;
    delta *= lift;
    // sum of p (dp - delta); the heaviest key's weight (from an eighth on), its place and a quarter of its score's derivative
    float rest = 0.0f, heaviest = 0.125f, bend = 1.0f;
    int heavy = -1;
    const float slope = a.slopes && there ? a.slopes[h] * kRecdLog2e : 0.0f;
    float from = there ? a.lse_in[at_row] * kRecdLog2e : 0.0f;
    if (from == -INFINITY)
        from = 0.0f;  // sees nothing
    from = capped.base - from;
    recd_f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; d++)
        o[d] = recd_f32x16{};
    typename S::Load ks, vs;
    if (a.d < DP)
        for (int b = 0; b < BUFS; b++) {
            ks.clear_behind(tid, kt[b], a.d);
            vs.clear_behind(tid, vt[b], a.d);
        }
    auto load = [&](int t) {
        const int64_t at = p.k0 + t * 32;
        ks.load_rows(tid, (const T *)a.k + at * a.k_stride + head * a.d, p.nk - t * 32, a.d, (uint32_t)a.k_stride * sizeof(T));
        vs.load_rows(tid, (const T *)a.v + at * a.v_stride + head * a.d, p.nk - t * 32, a.d, (uint32_t)a.v_stride * sizeof(T));
    };
    bool odd = false;  // something that is not finite in a tile at the edge
    if (t0 < t1)
        load(t0);
    for (int t = t0; t < t1; t++) {
        const int buf = BUFS == 1 ? 0 : t & 1;
        if constexpr (BUFS == 1)
            S::sync();
        ks.store(tid, kt[buf], a.d);
        vs.store(tid, vt[buf], a.d);
        const bool clear = t >= edge && any_wave<S::SHARED>(__any(ks.not_finite(tid)), says[t & 1], wave, lane);
        if (!S::SHARED || t < edge)
            S::sync();
        if (t + 1 < t1)
            load(t + 1);
        auto make_finite = [&]() {
            S::sync();
            kt[buf].make_finite(tid, S::LOADERS);
            S::sync();
            odd = true;
        };
        const int j0 = t * 32;
        if (S::SHARED && j0 >= wave_end) {
            if (clear)
                make_finite();
            continue;
        }
        recd_f32x16 s = {}, dp = {};
#pragma unroll
        for (int k = 0; k < KS; k++) {
            s = Mma::mul(kt[buf].rows(0, 16 * k, lane), qf[k], s);
            dp = Mma::mul(vt[buf].rows(0, 16 * k, lane), gf[k], dp);
        }
        if (clear)
            make_finite();
        // ds into s; where delta is still to settle first p, what it is the weight of in dp, and with a cap a quarter of the derivative in w
        recd_f32x16 w;
        auto score = [&](int r, float more) {
            float quarter = 1.0f;
            const float z = CAP ? capped.value(s[r] * to_cap, more, quarter) : s[r] * c + more;
            const float p = recd_exp2(z), of = dp[r] * lift - delta;
            s[r] = SETTLES ? p : p * of * quarter;
            dp[r] = of;
            w[r] = quarter;
        };
        auto finish = [&](auto registers) {
            constexpr int NR = registers.value;
            if (a.slopes) {
                const float far = (float)(pos - j0 - (lane >> 5));  // (whole numbers: positions may pass 2^24)
#pragma unroll
                for (int r = 0; r < NR; r++)
                    score(r, from - slope * fabsf(far - (float)recd_score_row(r, 0)));
            } else {
#pragma unroll
                for (int r = 0; r < NR; r++)
                    score(r, from);
            }
            if (j0 + 2 * NR > wave_full) {
                asm volatile("");  // a branch: only the tiles at the mask's edge pay for it
                const int to = lim - j0 - (lane >> 5);
#pragma unroll
                for (int r = 0; r < NR; r++)
                    if (recd_score_row(r, 0) >= to)
                        s[r] = dp[r] = w[r] = 0.0f;
            }
            if constexpr (SETTLES) {
                if (ONE && t1 == 1) {  // all keys at once: so is what is left of delta
#pragma unroll
                    for (int r = 0; r < NR; r++)
                        rest += s[r] * dp[r];
                    rest += __shfl_xor(rest, 32);
#pragma unroll
                    for (int r = 0; r < NR; r++)
                        s[r] *= CAP ? (dp[r] - rest) * w[r] : dp[r] - rest;
                    return;
                }
                float top = s[0];
#pragma unroll
                for (int r = 1; r < NR; r++)
                    top = fmaxf(top, s[r]);
                if (__any(top > heaviest))
#pragma unroll
                    for (int r = 0; r < NR; r++)
                        if (s[r] > heaviest) {
                            heaviest = s[r];
                            heavy = t * 16 + r;  // (its place below)
                            if (CAP)
                                bend = w[r];
                        }
#pragma unroll
                for (int r = 0; r < NR; r++) {
                    s[r] *= dp[r];
                    rest += s[r];
                    if (CAP)
                        s[r] *= w[r];
                }
            }
        };
        auto add = [&](auto registers) {
            constexpr int NR = registers.value;
            if constexpr (kHalf<T>) {
                const float f = keep_in_range<NR>(s, o);
                lift *= f;
                delta *= f;
                rest *= f;
            }
#pragma unroll
            for (int h = 0; h < NR / 8; h++) {
                const Frag sf = recd_sums_frag<T>(s, h);
#pragma unroll
                for (int d = 0; d < DT; d++)
                    o[d] = Mma::mul(kt[buf].columns(16 * h, 32 * d, lane), sf, o[d]);
            }
        };
        if (ONE && wave_end - j0 <= 16) {  // the other registers hold no key of the list
            finish(std::integral_constant<int, 8>{});
            add(std::integral_constant<int, 8>{});
        } else {
            finish(std::integral_constant<int, 16>{});
            add(std::integral_constant<int, 16>{});
        }
    }
    if (odd) {
        const T *keys = (const T *)a.k + p.k0 * a.k_stride + head * a.d;
        add_not_finite<false, T>(t0 > edge ? t0 * 32 : edge * 32, t1 * 32 < p.nk ? t1 * 32 : p.nk, a.d,
                                 [&](int j) { return keys + j * a.k_stride; }, [&](int j) { return j < lim; }, o, lane);
    }
    if constexpr (kHalf<T>) {
        scale_sums<DT>(o, inverse_power(lift));
        rest *= inverse_power(lift);
    }
    if constexpr (SETTLES) {
        heavy = heavy < 0 ? -1 : (heavy >> 4) * 32 + recd_score_row(heavy & 15, lane);
        // of the two halves of the wave, and of the phases in their order; of equal weights the first key
        auto take = [&](float more, float weight, float curve, int place) {
            rest += more;
            if (weight > heaviest || (weight == heaviest && (uint32_t)place < (uint32_t)heavy)) {
                heaviest = weight;
                bend = curve;
                heavy = place;
            }
        };
        if (!ONE || t1 > 1)
            take(__shfl_xor(rest, 32), __shfl_xor(heaviest, 32), __shfl_xor(bend, 32), __shfl_xor(heavy, 32));
        if constexpr (PHASES > 1) {
            of_phase[phase][0][lane] = rest;
            of_phase[phase][1][lane] = heaviest;
            of_phase[phase][2][lane] = bend;
            of_phase[phase][3][lane] = __int_as_float(heavy);
            __syncthreads();
            if (phase == 0)
                for (int ph = 1; ph < PHASES; ph++)
                    take(of_phase[ph][0][lane], of_phase[ph][1][lane], of_phase[ph][2][lane], __float_as_int(of_phase[ph][3][lane]));
        }
    }
    if constexpr (PHASES > 1) {
        static_assert(sizeof(lds) >= 64 * 16 * DT * sizeof(float));
        join_sums<DT, PHASES>(o, reinterpret_cast<float *>(&lds), 0, phase, lane);
    }
    if (phase)
        return;
    if (there && lane < 32)
        a.delta[at_row] = stored + rest;
    if (SETTLES && there && heavy >= 0)
        add_columns<T, DT>(o, -rest * bend, (const T *)a.k + (p.k0 + heavy) * a.k_stride + (int64_t)head * a.d, a.d, lane);
    if (there)
        store_columns<T, DT>((T *)a.gq + q_row * a.gq_stride + (int64_t)h * a.d, o, (CAP ? 4.0f : 1.0f) * a.scale, a.d, lane);
}

// Keys stay, queries and their gradients stream past.  What a score needs of its row stands in LDS in the order of
// the sums' registers: four neighbours are read at a time.
template <typename T, int DP, int KEPT, int PHASES, int CAP>
__global__ __launch_bounds__(64 * KEPT * PHASES, (kResident<T, DP, KEPT>)) void k_attention_grad_kv(Args a)
{
    using S = Shape<T, DP, KEPT, PHASES>;
    constexpr int KS = DP / 16, DT = DP / 32, BUFS = S::SHARED ? 2 : 1;
    using Mma = RecdMma<T>;
    using Frag = typename Mma::Frag;
    // Wide heads with two phases: the kept keys and values stay in LDS, read as operands from there, as the registers
    // hold two sums of the head's width besides.
    constexpr bool IN_LDS = S::SHARED && PHASES > 1;
    __shared__ struct {
        typename S::Tile q[S::OWN][BUFS], g[S::OWN][BUFS];
        RecdTile<T, IN_LDS ? 32 * KEPT : 1, DP> k, v;
        alignas(16) float from[S::OWN][BUFS][S::ROWS], delta[S::OWN][BUFS][S::ROWS], slope[S::OWN][BUFS][S::ROWS];
        alignas(16) float pos[S::OWN][BUFS][S::ROWS];
        alignas(16) int lim[S::OWN][BUFS][S::ROWS];
    } lds;
    __shared__ int says[2][KEPT * PHASES];
    Problem p;
    int head, head_end, tile, split;
    if (!find_tile(a, p, head, head_end, tile, split))
        return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kept = wave % KEPT, phase = wave / KEPT;
    const int tid = S::SHARED ? threadIdx.x : lane, own = S::SHARED ? 0 : phase;
    typename S::Tile *const qt = lds.q[own], *const gt = lds.g[own];
    const auto row_from = lds.from[own], row_delta = lds.delta[own], row_slope = lds.slope[own];
    const auto row_pos = lds.pos[own];
    const auto row_lim = lds.lim[own];
    const int first = tile * 32 * KEPT;
    if (first >= p.nk)
        return;
    const int j0 = first + 32 * kept, j = j0 + (lane & 31);
    const bool there = j < p.nk;
    const float jf = (float)(j - first);  // positions count from the block's first key, as whole numbers may pass 2^24
    const int H = a.G * a.group;
    Frag kf[IN_LDS ? 1 : KS], vf[IN_LDS ? 1 : KS];
    const int kept_at = IN_LDS ? (32 * kept + (lane & 31)) * lds.k.LD + (lane >> 5) * 8 : 0;
#pragma unroll
    for (int k = 0; k < KS; k++) {
        const int i = IN_LDS ? 0 : k;
        if (IN_LDS && k % PHASES != phase)
            continue;  // the phases share the writing
        kf[i] = recd_row_frag<T>((const T *)a.k + (p.k0 + j) * a.k_stride + (int64_t)head * a.d, 16 * k, a.d, there, lane);
        vf[i] = recd_row_frag<T>((const T *)a.v + (p.k0 + j) * a.v_stride + (int64_t)head * a.d, 16 * k, a.d, there, lane);
        if constexpr (IN_LDS) {
            *reinterpret_cast<Frag *>(lds.k.at + kept_at + 16 * k) = kf[0];
            *reinterpret_cast<Frag *>(lds.v.at + kept_at + 16 * k) = vf[0];
        }
    }
    recd_f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; d++)
        dk[d] = dv[d] = recd_f32x16{};
    // probabilities are held 2^kLiftP larger, by their exponents; ds by that and the rest of its lift
    float lift = kHalf<T> ? kFirstLift * 0x1p-15f : 1.0f;
    const float c = a.scale * kRecdLog2e;
    const Capped<CAP> capped(a.cap);
    const float to_cap = CAP ? 2.0f * kRecdLog2e * a.scale / a.cap : 0.0f;
    // the first row that sees the block's first key
    int from_row = 0;
    if (p.causal && p.prefix <= first && first > p.pos0)
        from_row = (int)((int64_t)(first - p.pos0) * a.group < p.rows ? (first - p.pos0) * a.group : p.rows);
    // (a wave that streams for itself takes its part of the tiles, a phase of a block its 32 rows of every tile)
    const int tiles = (p.rows + S::ROWS - 1) / S::ROWS, from_tile = from_row / S::ROWS, n_tiles = tiles - from_tile;
    const int t0 = S::SHARED ? from_tile : from_tile + n_tiles * phase / PHASES;
    const int t1 = S::SHARED ? tiles : from_tile + n_tiles * (phase + 1) / PHASES;
    const int sub = S::SHARED ? 32 * phase : 0;
    // rows from `whole_row` on see all of the block's keys; tiles with earlier ones, and a last one that is filled up, are at the edge
    // (a wave that has few tiles looks all of them through)
    const int keys_end = first + 32 * KEPT < p.nk ? first + 32 * KEPT : p.nk;
    int whole_row = 0;
    if (p.causal && p.prefix < keys_end && keys_end - 1 > p.pos0)
        whole_row = (int)((int64_t)(keys_end - 1 - p.pos0) * a.group < p.rows ? (keys_end - 1 - p.pos0) * a.group : p.rows);
    auto at_edge = [&](int t) { return KEPT * PHASES == 1 || t * S::ROWS < whole_row || (t + 1) * S::ROWS > p.rows; };
    bool odd = false;  // something that is not finite in a tile at the edge
    typename S::Load qs, gs;
    if (a.d < DP)
        for (int b = 0; b < BUFS; b++) {
            qs.clear_behind(tid, qt[b], a.d);
            gs.clear_behind(tid, gt[b], a.d);
        }
    float n_from = 0.0f, n_delta = 0.0f, n_slope = 0.0f;
    float n_pos = 0.0f;
    int n_lim = 0;
    auto load = [&](int t) {
        // the tile's first row is head `odd` of its query's; row r is then query (odd + r) / group from there
        const int row = t * S::ROWS, q_first = p.query(row, a.group), odd = row - q_first * a.group;
        auto query_of = [&](int r) { return a.group == 1 ? r : (int)__umulhi(odd + r, a.by_group); };
        auto rows_at = [&](uint32_t stride) {
            return [=](int r) {
                const int query = query_of(r);
                return (uint32_t)__umul24(query, stride) + (uint32_t)((odd + r - query * a.group) * a.d * (int)sizeof(T));
            };
        };
        const int64_t at = p.q0 + q_first;
        qs.load(tid, (const T *)a.q + at * a.q_stride + head * a.group * a.d, p.rows - row, a.d,
                rows_at((uint32_t)a.q_stride * sizeof(T)));
        gs.load(tid, (const T *)a.g + (at * H + head * a.group) * a.d, p.rows - row, a.d, rows_at(H * a.d * sizeof(T)));
        n_from = n_delta = n_slope = 0.0f;
        n_pos = 0.0f;
        n_lim = 0;
        if (tid < S::ROWS && row + tid < p.rows) {
            const int in = query_of(tid), query = q_first + in, h = head * a.group + odd + tid - in * a.group;
            n_from = a.lse_in[(p.q0 + query) * H + h] * kRecdLog2e;
            n_from = (n_from == -INFINITY ? 0.0f : -n_from) + (kLiftP<T> + capped.base);
            n_delta = a.delta[(p.q0 + query) * H + h];
            n_slope = a.slopes ? a.slopes[h] * kRecdLog2e : 0.0f;
            n_lim = p.limit_at(query);
            n_pos = (float)(p.pos0 + query - first);
        }
    };
    if (t0 < t1)
        load(t0);
    for (int t = t0; t < t1; t++) {
        const int buf = BUFS == 1 ? 0 : t & 1;
        if constexpr (BUFS == 1)
            S::sync();
        qs.store(tid, qt[buf], a.d);
        gs.store(tid, gt[buf], a.d);
        if (tid < S::ROWS) {
            const int i = recd_product_row(tid);
            row_from[buf][i] = n_from;
            row_delta[buf][i] = n_delta;
            row_slope[buf][i] = n_slope;
            row_lim[buf][i] = n_lim;
            row_pos[buf][i] = n_pos;
        }
        const bool clear = at_edge(t) && any_wave<S::SHARED>(__any(qs.not_finite(tid) | gs.not_finite(tid)), says[t & 1], wave, lane);
        if (!S::SHARED || !at_edge(t))
            S::sync();
        if (t + 1 < t1)
            load(t + 1);
        auto make_finite = [&]() {
            S::sync();
            qt[buf].make_finite(tid, S::LOADERS);
            gt[buf].make_finite(tid, S::LOADERS);
            S::sync();
            odd = true;
        };
        const int row0 = t * S::ROWS + sub;
        const bool whole = row0 + 32 <= p.rows;
        // (tile row 31 is the product's row 31, and limits do not fall: what it does not see, no row sees)
        if (j0 >= p.nk || row0 >= p.rows || (whole && __builtin_amdgcn_readfirstlane(row_lim[buf][sub + 31]) <= j0)) {
            if (S::SHARED && clear)
                make_finite();
            continue;
        }
        recd_f32x16 s = {}, dp = {};
#pragma unroll
        for (int k = 0; k < KS; k++) {
            Frag key, value;
            if constexpr (IN_LDS) {
                key = *reinterpret_cast<const Frag *>(lds.k.at + kept_at + 16 * k);
                value = *reinterpret_cast<const Frag *>(lds.v.at + kept_at + 16 * k);
            } else {
                key = kf[k];
                value = vf[k];
            }
            s = Mma::mul(qt[buf].rows(sub, 16 * k, lane), key, s);
            dp = Mma::mul(gt[buf].rows(sub, 16 * k, lane), value, dp);
        }
        if (clear)
            make_finite();
        auto score = [&](int r, float more, float delta) {
            float quarter = 1.0f;
            const float z = CAP ? capped.value(s[r] * to_cap, more, quarter) : s[r] * c + more;
            s[r] = recd_exp2(z);
            dp[r] = s[r] * (dp[r] - delta) * (kHalf<T> ? quarter * lift : quarter);
        };
        if (a.slopes) {
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int row = sub + recd_sums_row(r, lane);
                const recd_f32x4 from = *reinterpret_cast<const recd_f32x4 *>(&row_from[buf][row]);
                const recd_f32x4 delta = *reinterpret_cast<const recd_f32x4 *>(&row_delta[buf][row]);
                const recd_f32x4 slope = *reinterpret_cast<const recd_f32x4 *>(&row_slope[buf][row]);
                const recd_f32x4 pos = *reinterpret_cast<const recd_f32x4 *>(&row_pos[buf][row]);
#pragma unroll
                for (int q = 0; q < 4; q++)
                    score(r + q, from[q] - slope[q] * fabsf(pos[q] - jf), delta[q]);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int row = sub + recd_sums_row(r, lane);
                const recd_f32x4 from = *reinterpret_cast<const recd_f32x4 *>(&row_from[buf][row]);
                const recd_f32x4 delta = *reinterpret_cast<const recd_f32x4 *>(&row_delta[buf][row]);
#pragma unroll
                for (int q = 0; q < 4; q++)
                    score(r + q, from[q], delta[q]);
            }
        }
        // (tile row 0 is the product's row 0, and limits do not fall: what its rows all see, the others see)
        if (!whole || __builtin_amdgcn_readfirstlane(row_lim[buf][sub]) < j0 + 32) {
            asm volatile("");
#pragma unroll
            for (int r = 0; r < 16; r++)
                if (j >= row_lim[buf][sub + recd_sums_row(r, lane)])
                    s[r] = dp[r] = 0.0f;
        }
        if constexpr (kHalf<T>)
            lift *= keep_in_range<16>(dp, dk);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const Frag pf = recd_sums_frag<T>(s, h), sf = recd_sums_frag<T>(dp, h);
#pragma unroll
            for (int d = 0; d < DT; d++) {
                dv[d] = Mma::mul(gt[buf].columns(sub + 16 * h, 32 * d, lane), pf, dv[d]);
                dk[d] = Mma::mul(qt[buf].columns(sub + 16 * h, 32 * d, lane), sf, dk[d]);
            }
        }
    }
    if (odd) {
        auto at = [&](const void *x, int64_t stride) {
            return [=, &p, &a](int row) {
                const int query = p.query(row, a.group), h = head * a.group + row - query * a.group;
                return (const T *)x + (p.q0 + query) * stride + (int64_t)h * a.d;
            };
        };
        auto sees = [&](int row) { return j < p.limit(row, a.group); };
#pragma unroll 1
        for (int t = t0; t < t1; t++) {
            const int s0 = t * S::ROWS + sub, s1 = s0 + 32 < p.rows ? s0 + 32 : p.rows;
            if (!at_edge(t))
                continue;
            add_not_finite<false, T>(s0, s1, a.d, at(a.q, a.q_stride), sees, dk, lane);
            add_not_finite<true, T>(s0, s1, a.d, at(a.g, (int64_t)H * a.d), sees, dv, lane);
        }
    }
    if constexpr (kHalf<T>)
        scale_sums<DT>(dk, inverse_power(lift) * 0x1p-15f);
    if constexpr (PHASES > 1) {
        static_assert(sizeof(lds) >= KEPT * 64 * 16 * DT * sizeof(float));
        join_sums<DT, PHASES>(dk, reinterpret_cast<float *>(&lds), kept, phase, lane);
        join_sums<DT, PHASES>(dv, reinterpret_cast<float *>(&lds), kept, phase, lane);
    }
    if (phase)
        return;
    if (there) {
        store_columns<T, DT>((T *)a.gk + (p.k0 + j) * a.gk_stride + (int64_t)head * a.d, dk, (CAP ? 4.0f : 1.0f) * a.scale, a.d,
                             lane);
        store_columns<T, DT>((T *)a.gv + (p.k0 + j) * a.gv_stride + (int64_t)head * a.d, dv, recd_exp2(-kLiftP<T>), a.d, lane);
    }
}

// Offsets that do not rise from 0 to the number of rows, or pass the caller's bound of a list's length.
__global__ void k_validate_list_offsets(int64_t lists, int64_t rows, int64_t most, const int64_t *offsets, int *err)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i <= lists; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t at = offsets[i];
        if ((i == 0 && at != 0) || (i == lists && at != rows))
            atomicOr(err, 1);
        if (i < lists && (offsets[i + 1] < at || offsets[i + 1] - at > most))
            atomicOr(err, 1);
    }
}

recd_status check_attention(recd_ctx *ctx, const recd_attention *a, const void *q, const void *k, const void *v)
{
    if (!ctx)
        return RECD_EINVAL;
    if (!a)
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if ((int)a->dtype < 0 || (int)a->dtype > 2)
        return recd_fail(ctx, RECD_EINVAL, "unknown dtype");
    if (a->heads <= 0 || a->kv_heads <= 0 || a->heads % a->kv_heads != 0 || a->heads > 4096)
        return recd_fail(ctx, RECD_EINVAL, "heads=%d must be a multiple of kv_heads=%d, and at most 4096", a->heads, a->kv_heads);
    const int64_t es = (int64_t)elem_size(a->dtype);
    if (a->head_dim <= 0 || a->head_dim > RECD_MAX_HEAD_DIM || a->head_dim * es % 16 != 0)
        return recd_fail(ctx, RECD_EINVAL, "head_dim=%d: a head's bytes must be a multiple of 16, and head_dim at most %d",
                         a->head_dim, RECD_MAX_HEAD_DIM);
    if (a->lists < 0 || a->max_q < 0 || a->max_k < 0 || a->q_rows < 0 || a->k_rows < 0)
        return recd_fail(ctx, RECD_EINVAL, "lists, max_q, max_k, q_rows or k_rows < 0");
    // (rows are counted in 32 bits, up to a tile of every split behind the last one)
    const int64_t most = RECD_MAX_LIST;
    if (a->lists > most / 2 || a->max_q > most / a->heads || a->max_k > most)
        return recd_fail(ctx, RECD_EINVAL, "lists, max_q * heads or max_k too large (%lld, %lld, %lld)", (long long)(most / 2),
                         (long long)most, (long long)most);
    if (!(a->softcap >= 0.0f) || a->softcap == INFINITY)
        return recd_fail(ctx, RECD_EINVAL, "softcap must be 0 (none) or positive");
    if (a->prefix && !a->causal)
        return recd_fail(ctx, RECD_EINVAL, "prefix needs causal");
    if (a->lists == 0 ? a->q_rows || a->k_rows : !a->q_offsets || !a->k_offsets)
        return recd_fail(ctx, RECD_EINVAL, "rows without lists, or null offsets");
    if ((a->q_rows && !q) || (a->k_rows && (!k || !v)))
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (a->q_stride < (int64_t)a->heads * a->head_dim || a->k_stride < (int64_t)a->kv_heads * a->head_dim ||
        a->v_stride < (int64_t)a->kv_heads * a->head_dim)
        return recd_fail(ctx, RECD_EINVAL, "a stride is less than a row");
    if (a->q_stride * es >= 1 << 24 || a->k_stride * es >= 1 << 24 || a->v_stride * es >= 1 << 24)
        return recd_fail(ctx, RECD_EINVAL, "rows 16 MiB apart and more");
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v) % 16 || (a->q_stride | a->k_stride | a->v_stride) * es % 16)
        return recd_fail(ctx, RECD_EINVAL, "q, k, v and their strides must be aligned to 16 bytes");
    return RECD_OK;
}

recd_status validate_lists(recd_ctx *ctx, const recd_attention *a)
{
    ctx->plan.valid = false;
    RECD_TRY(recd_reserve(ctx, RECD_VALIDATE_BYTES));
    int *err = reinterpret_cast<int *>(ctx->ws);
    RECD_HIP(ctx, hipMemsetAsync(err, 0, sizeof(int), ctx->stream));
    hipLaunchKernelGGL(k_validate_list_offsets, dim3(64), dim3(256), 0, ctx->stream, a->lists, a->q_rows, a->max_q,
                       a->q_offsets, err);
    hipLaunchKernelGGL(k_validate_list_offsets, dim3(64), dim3(256), 0, ctx->stream, a->lists, a->k_rows, a->max_k,
                       a->k_offsets, err);
    RECD_HIP(ctx, hipGetLastError());
    ctx->host_pinned[0] = 0;
    RECD_HIP(ctx, hipMemcpyAsync(ctx->host_pinned, err, sizeof(int), hipMemcpyDeviceToHost, ctx->stream));
    RECD_HIP(ctx, hipStreamSynchronize(ctx->stream));
    if ((int)ctx->host_pinned[0])
        return recd_fail(ctx, RECD_EBOUNDS, "offsets do not rise from 0 to the rows, or a list is longer than its bound");
    return RECD_OK;
}

Args common_args(const recd_attention *d, const void *q, const void *k, const void *v)
{
    Args a{};
    a.G = d->kv_heads;
    a.group = d->heads / d->kv_heads;
    a.d = d->head_dim;
    a.by_group = (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group);
    a.lists = d->lists;
    a.splits = 1;
    a.q_offsets = d->q_offsets;
    a.k_offsets = d->k_offsets;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = d->q_stride;
    a.k_stride = d->k_stride;
    a.v_stride = d->v_stride;
    a.scale = d->scale;
    a.cap = d->softcap;
    a.slopes = d->slopes;
    a.prefix = d->prefix;
    a.causal = d->causal != 0;
    a.part_rows = d->q_rows * d->heads;
    a.last_first = true;
    a.heads = 1;
    return a;
}

enum Which { FORWARD, GRAD_Q, GRAD_KV };

// How a kernel's blocks divide their tiles: one wave; one group of 32 kept rows in phases; four groups (and, for the wide
// 16-bit heads of the gradients by keys and values, two phases).
enum Division { ONE_WAVE, PHASES, GROUPS };

// How the tiles of one side are listed: the kept rows of a tile, and slots.
struct Tiling {
    Division division;
    int R, tiles_per_list;
    int64_t slots;
    bool table;
};

// Lists of few rows (here and on the other side) give every tile to a wave of its own; so many tiles that four groups in a
// block fill the card share what they stream; in between a tile's streamed rows are divided among the waves. In us,
// forward and backward, bf16, lists that attend to themselves under the causal mask, one wave / phases / groups:
//   2000 lists of 80 rows, 4 heads of 32       43, 134 / 127, 262 / 48, 145
//   64 lists of 300, 4 heads on 2 of 64        18, 50 / 32, 66 / 14, 50
//   8 lists of up to 4096, 8 on 4 heads of 128  317, 883 / 342, 905 / 135, 423
// and single rows, 8 heads on 2 of 64: 2000 lists of 100 keys 24 / 44 / 35, 37 lists of up to 16 384 53 / 39 / 58.
// Where phases give way to groups: a block of phases holds the parts of four waves in the LDS that a block of groups
// shares, and wide heads leave fewer of them to a compute unit, so the number of groups' blocks from which the groups
// are faster falls with the width. Phases against groups, gradients by keys at lists of 400 rows, in us:
//   bf16, heads of 32:   256 blocks 11 / 19, 512 blocks 18 / 20, 768 blocks 24 / 21
//   bf16, heads of 64:   256 blocks 19 / 24, 512 blocks 34 / 27
//   bf16, heads of 128:  64 blocks 19 / 23, 128 blocks 27 / 24, 256 blocks 48 / 26
//   fp32, heads of 32:   256 blocks 28 / 42, 512 blocks 51 / 53, and the forward pass 22 / 24 and 35 / 33
//   fp32, heads of 64:   256 blocks 60 / 71, 512 blocks 112 / 90, and the forward pass 42 / 39 and 77 / 57
Tiling tiling(const recd_ctx *ctx, const recd_attention *d, int64_t rows, int64_t most, int group, int64_t others,
              int64_t most_others)
{
    Tiling t;
    // groups' blocks, each counted for as much as its list is long beside the longest, which they wait for
    const double blocks = (double)(rows * group) / 128 * d->kv_heads * ((double)others / ((double)d->lists * (double)(most_others > 0 ? most_others : 1)));
    const bool f32 = d->dtype == RECD_F32, few = most * group <= 64 || rows * group <= 48 * d->lists;
    const bool wide = f32 && d->head_dim > 64;  // tiles of 17 KB: phases would leave two waves to a compute unit
    const int quarters = d->head_dim <= 32 ? (f32 ? 6 : 8) : d->head_dim <= 64 ? (f32 ? 4 : 5) : 2;
    if (few && (wide || most_others <= 128 || others <= 64 * d->lists))
        t.division = ONE_WAVE;
    else if (!wide && (few || 4 * blocks < (double)quarters * ctx->num_cu))
        t.division = PHASES;
    else
        t.division = GROUPS;
    t.R = t.division == GROUPS ? 128 : 32;
    const int64_t per = (most * group + t.R - 1) / t.R;
    t.slots = rows * group / t.R + d->lists;
    t.table = d->lists * per > t.slots;
    if (!t.table)
        t.slots = d->lists * per;
    t.tiles_per_list = (int)(per > 0 ? per : 1);
    return t;
}

int log2_of(int n)
{
    int l = 0;
    while ((1 << l) < n)
        l++;
    return l;
}

int64_t blocks_of(int64_t slots, int splits, int G, int heads) { return (slots * splits + 7) / 8 * 8 * ((G + heads - 1) / heads); }
unsigned grid_of(const Args &a) { return (unsigned)blocks_of(a.slots, a.splits, a.G, a.heads); }

// A launch holds less than 2^32 threads.
bool launch_holds(const Tiling &t, int splits, int G, int heads)
{
    const int threads = t.division == ONE_WAVE ? 64 : t.division == PHASES ? 256 : 512;
    return blocks_of(t.slots, splits, G, heads) < ((int64_t)1 << 32) / threads;
}

// Key heads that a block of one wave goes through, the next head's rows on their way while it works at one: as many as
// leave four rounds of waves (about twelve a compute unit at a time).  Forward, with and without, in us: 8192 lists of up to
// 100 rows, 4 heads of 32 bf16 46.1 / 47.4; 40 000 of them 214 / 225; 20 000 of 20 rows, 8 heads of 64 388 / 437; 20 000 of 30,
// fp32 274 / 311; but 20 000 single rows against 100 keys each 709 / 682.
int heads_at_once(const recd_ctx *ctx, const Tiling &t, int G, int64_t lists)
{
    int heads = 1;
    while (t.division == ONE_WAVE && heads < G && (t.slots - lists / 2) * ((G + 2 * heads - 1) / (2 * heads)) >= (int64_t)ctx->num_cu * 48)
        heads *= 2;
    return heads;
}


template <typename T, int DP, int CAP> void launch_one(Which w, const Args &a, Division v, hipStream_t st)
{
    constexpr int KV = sizeof(T) == 2 && DP > 64 ? 2 : 1;
    constexpr bool WIDE = sizeof(T) == 4 && DP > 64;
    const dim3 grid(grid_of(a));
#define RECD_LAUNCH(kernel, kept, phases) \
    hipLaunchKernelGGL((kernel<T, DP, kept, phases, CAP>), grid, dim3(64 * kept * phases), 0, st, a)
    if (w == FORWARD) {
        if (v == ONE_WAVE)
            hipLaunchKernelGGL((k_attention_one<T, DP, CAP>), grid, dim3(64), 0, st, a);
        else if (v == PHASES) {
            if constexpr (!WIDE)
                RECD_LAUNCH(k_attention, 1, 4);
        } else
            RECD_LAUNCH(k_attention, 4, 1);
    } else if (w == GRAD_Q) {
        if (v == ONE_WAVE)
            RECD_LAUNCH(k_attention_grad_q, 1, 1);
        else if (v == PHASES) {
            if constexpr (!WIDE)
                RECD_LAUNCH(k_attention_grad_q, 1, 4);
        } else
            RECD_LAUNCH(k_attention_grad_q, 4, 1);
    } else {
        if (v == ONE_WAVE)
            RECD_LAUNCH(k_attention_grad_kv, 1, 1);
        else if (v == PHASES) {
            if constexpr (!WIDE)
                RECD_LAUNCH(k_attention_grad_kv, 1, 4);
        } else
            RECD_LAUNCH(k_attention_grad_kv, 4, KV);
    }
#undef RECD_LAUNCH
}

template <typename T, int DP> void launch_width(Which w, const Args &a, Division v, hipStream_t st)
{
    if (a.cap == 0.0f)
        launch_one<T, DP, NO_CAP>(w, a, v, st);
    else if (sizeof(T) == 4 || a.cap > 256.0f)
        launch_one<T, DP, CAP_WIDE>(w, a, v, st);
    else
        launch_one<T, DP, sizeof(T) == 2 ? CAP_16 : CAP_WIDE>(w, a, v, st);
}

template <typename T> void launch(Which w, const Args &a, Division v, hipStream_t st)
{
    if (a.slots * a.splits == 0)
        return;
    if (a.d <= 32)
        launch_width<T, 32>(w, a, v, st);
    else if (a.d <= 64)
        launch_width<T, 64>(w, a, v, st);
    else
        launch_width<T, 128>(w, a, v, st);
}

// Lists the tiles of up to two sides that have a table.
void launch_tiles(const recd_attention *d, const Side *sides, int n, hipStream_t st)
{
    if (n == 0)
        return;
    const Side &one = sides[0], &two = sides[n - 1];
    if (d->lists <= kMostSorted && one.slots < ((int64_t)1 << 30) && two.slots < ((int64_t)1 << 30))
        hipLaunchKernelGGL(k_attention_tiles_by_work, dim3(n), dim3(1024), 0, st, (int)d->lists, d->causal != 0, d->q_offsets,
                           d->k_offsets, d->prefix, one, two);
    else
        hipLaunchKernelGGL(k_attention_tiles, dim3((unsigned)((d->lists + 255) / 256), n), dim3(256), 0, st, d->lists, d->q_offsets,
                           d->k_offsets, one, two);
}

// How a forward call is cut, into `a`.
Tiling forward_tiling(const recd_ctx *ctx, const recd_attention *d, Args &a)
{
    const Tiling t = tiling(ctx, d, d->q_rows, d->max_q, a.group, d->k_rows, d->max_k);
    a.slots = t.slots;
    a.tiles_per_list = t.tiles_per_list;
    a.heads = heads_at_once(ctx, t, a.G, d->lists);
    // Few tiles: a tile's keys are split over blocks, at least 512 keys each (one query against 30 000 keys 14 us, with 256
    // 14, with 1024 17; 8 against 16 384 each 20.7, 22.3, 20.5), until two blocks a compute unit are at work (37 queries
    // against up to 16 384 keys 43 us, with one 46, with four 46); tiles of one wave eight.
    const int64_t blocks = (int64_t)ctx->num_cu * (t.division == ONE_WAVE ? 8 : 2), have = t.slots * a.G > 0 ? t.slots * a.G : 1;
    int64_t splits = (blocks + have - 1) / have;
    if (splits > d->max_k / 512)
        splits = d->max_k / 512;
    if (splits > kMostSplits)
        splits = kMostSplits;
    a.splits = (int)(splits < 1 ? 1 : splits);
    return t;
}

void carve_forward(WsCarver &c, const Tiling &t, Args &a, int2 *&tiles)
{
    tiles = t.table ? c.take<int2>(t.slots) : nullptr;
    a.part_m = a.splits > 1 ? c.take<float>(a.splits * a.part_rows) : nullptr;
    a.part_l = a.splits > 1 ? c.take<float>(a.splits * a.part_rows) : nullptr;
    a.part_o = a.splits > 1 ? c.take<float>(a.splits * a.part_rows * a.d) : nullptr;
}

// The tiles by queries and by keys of a backward call.
struct BackwardTiling {
    Tiling q, k;

    BackwardTiling(const recd_ctx *ctx, const recd_attention *d, const Args &a)
        : q(tiling(ctx, d, d->q_rows, d->max_q, a.group, d->k_rows, d->max_k)),
          k(tiling(ctx, d, d->k_rows, d->max_k, 1, d->q_rows * a.group, d->max_q * a.group))
    {
    }
    void carve(WsCarver &c, Args &a, int2 *&tiles_q, int2 *&tiles_k) const
    {
        tiles_q = q.table ? c.take<int2>(q.slots) : nullptr;
        tiles_k = k.table ? c.take<int2>(k.slots) : nullptr;
        a.delta = c.take<float>(a.part_rows);
    }
};

} // namespace

extern "C" {

recd_status recd_list_attention_workspace_bytes(int device, const recd_attention *sizes, size_t *out_bytes)
{
    recd_ctx c;
    if (!sizes || !out_bytes)
        return RECD_EINVAL;
    static const int64_t nothing = 0;
    recd_attention d = *sizes;  // with what the check asks for in the place of pointers and strides
    d.q_offsets = d.k_offsets = &nothing;
    d.q_stride = (int64_t)d.heads * d.head_dim;
    d.k_stride = d.v_stride = (int64_t)d.kv_heads * d.head_dim;
    d.prefix = nullptr;
    const void *some = reinterpret_cast<const void *>(16);
    RECD_TRY(check_attention(&c, &d, some, some, some));
    RECD_TRY(recd_sizing_context(&c, device));
    *out_bytes = RECD_VALIDATE_BYTES;
    if (d.lists == 0)
        return RECD_OK;
    Args a = common_args(&d, some, some, some);
    int2 *tiles, *tiles_k;
    if (d.q_rows > 0) {
        WsCarver forward(nullptr);
        const Tiling t = forward_tiling(&c, &d, a);
        carve_forward(forward, t, a, tiles);
        *out_bytes = larger(*out_bytes, forward.off);
    }
    WsCarver backward(nullptr);
    BackwardTiling(&c, &d, a).carve(backward, a, tiles, tiles_k);
    *out_bytes = larger(*out_bytes, backward.off);
    return RECD_OK;
}

recd_status recd_list_attention(recd_ctx *ctx, const recd_attention *d, const void *q, const void *k, const void *v, void *out,
                                float *lse)
{
    RECD_TRY(check_attention(ctx, d, q, k, v));
    if (d->q_rows && !out)
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if ((uintptr_t)out % 16)
        return recd_fail(ctx, RECD_EINVAL, "out must be aligned to 16 bytes");
    if (d->lists == 0 || d->q_rows == 0)
        return RECD_OK;
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    if (ctx->validate)
        RECD_TRY(validate_lists(ctx, d));
    Args a = common_args(d, q, k, v);
    a.out = out;
    a.lse = lse;
    const Tiling t = forward_tiling(ctx, d, a);
    if (!launch_holds(t, a.splits, a.G, a.heads))
        return recd_fail(ctx, RECD_EINVAL, "more tiles than a launch holds");
    int2 *tiles;
    WsCarver size(nullptr);
    carve_forward(size, t, a, tiles);
    if (size.off) {
        ctx->plan.valid = false;  // tiles and parts overwrite the workspace a backward plan would live in
        RECD_TRY(recd_reserve(ctx, size.off));
    }
    WsCarver c(ctx->ws);
    carve_forward(c, t, a, tiles);
    a.tiles = tiles;
    const Side side{t.slots, a.group, t.R, false, tiles};
    launch_tiles(d, &side, t.table ? 1 : 0, ctx->stream);
    recd_with_type(d->dtype, [&](auto e) {
        using T = decltype(e);
        launch<T>(FORWARD, a, t.division, ctx->stream);
        if (a.splits > 1) {
            const int dlog = log2_of(a.d / 4);
            if (a.splits > 8)
                hipLaunchKernelGGL((k_attention_join_many<T>), dim3((unsigned)a.part_rows), dim3(256), 0, ctx->stream, a.part_rows,
                                   a.d, dlog, a.splits, a.part_m, a.part_l, a.part_o, (T *)out, lse);
            else
                hipLaunchKernelGGL((k_attention_join<T>), dim3((unsigned)(((a.part_rows << dlog) + 255) / 256)), dim3(256), 0,
                                   ctx->stream, a.part_rows, a.d, dlog, a.splits, a.part_m, a.part_l, a.part_o, (T *)out, lse);
        }
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

recd_status recd_list_attention_backward(recd_ctx *ctx, const recd_attention *d, const void *q, const void *k, const void *v,
                                         const void *out, const float *lse, const void *grad_out, void *grad_q, void *grad_k,
                                         void *grad_v, int64_t grad_q_stride, int64_t grad_k_stride, int64_t grad_v_stride)
{
    RECD_TRY(check_attention(ctx, d, q, k, v));
    if ((d->q_rows && (!out || !lse || !grad_out || !grad_q)) || (d->k_rows && (!grad_k || !grad_v)))
        return recd_fail(ctx, RECD_EINVAL, "null pointer argument");
    if (grad_q_stride < (int64_t)d->heads * d->head_dim || grad_k_stride < (int64_t)d->kv_heads * d->head_dim ||
        grad_v_stride < (int64_t)d->kv_heads * d->head_dim)
        return recd_fail(ctx, RECD_EINVAL, "a stride is less than a row");
    if (((uintptr_t)out | (uintptr_t)grad_out | (uintptr_t)grad_q | (uintptr_t)grad_k | (uintptr_t)grad_v) % 16 ||
        (grad_q_stride | grad_k_stride | grad_v_stride) * (int64_t)elem_size(d->dtype) % 16)
        return recd_fail(ctx, RECD_EINVAL, "out, the gradients and their strides must be aligned to 16 bytes");
    if (d->lists == 0)
        return RECD_OK;
    RECD_HIP(ctx, hipSetDevice(ctx->device));
    if (ctx->validate)
        RECD_TRY(validate_lists(ctx, d));
    Args a = common_args(d, q, k, v);
    a.out_in = out;
    a.lse_in = lse;
    a.g = grad_out;
    a.gq = grad_q;
    a.gk = grad_k;
    a.gv = grad_v;
    a.gq_stride = grad_q_stride;
    a.gk_stride = grad_k_stride;
    a.gv_stride = grad_v_stride;
    const BackwardTiling tilings(ctx, d, a);
    const Tiling &tq = tilings.q, &tk = tilings.k;
    if (!launch_holds(tq, 1, a.G, 1) || !launch_holds(tk, 1, a.G, 1))
        return recd_fail(ctx, RECD_EINVAL, "more tiles than a launch holds");
    int2 *tiles_q, *tiles_k;
    WsCarver size(nullptr);
    tilings.carve(size, a, tiles_q, tiles_k);
    ctx->plan.valid = false;
    RECD_TRY(recd_reserve(ctx, size.off));
    WsCarver c(ctx->ws);
    tilings.carve(c, a, tiles_q, tiles_k);
    hipStream_t st = ctx->stream;
    Side sides[2];
    int listed = 0;
    if (tq.table)
        sides[listed++] = Side{tq.slots, a.group, tq.R, false, tiles_q};
    if (tk.table)
        sides[listed++] = Side{tk.slots, 1, tk.R, true, tiles_k};
    launch_tiles(d, sides, listed, st);
    recd_with_type(d->dtype, [&](auto e) {
        using T = decltype(e);
        if (d->q_rows) {
            a.tiles = tiles_q;
            a.slots = tq.slots;
            a.tiles_per_list = tq.tiles_per_list;
            launch<T>(GRAD_Q, a, tq.division, st);
        }
        a.tiles = tiles_k;
        a.last_first = false;
        a.slots = tk.slots;
        a.tiles_per_list = tk.tiles_per_list;
        if (d->k_rows)
            launch<T>(GRAD_KV, a, tk.division, st);
    });
    RECD_HIP(ctx, hipGetLastError());
    return RECD_OK;
}

} // extern "C"
