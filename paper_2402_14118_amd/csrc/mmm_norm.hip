// The norms around a block with its gate and residual (mmm_block_norm), their gradients, and the gradient through the epilogue of
// the multiplication: the operators of a residual block that touch every element a few times.
//
//     v = norm_post(y) w + b        h' = alpha h + g v        n = norm_pre(h') w' + b'
//
// Each reads its inputs and writes its outputs once.  A workgroup keeps a row in registers, eight neighbours (16 bytes of a 16-bit type) per lane and
// piece; both norms, gate and residual work on that.  Sums of a row: lanes by cross-lane moves, waves through LDS, in a fixed order.  The variance is
// that of the centred row, which stands there anyway, not a difference of two sums.
//
// What bounds them.  The norms up to 8192 wide, and the gradient through the epilogue of many elements: HBM (2048 x 4096 bf16 14.0 us, 67 MB at 4.8 TB/s; wider
// than 4096 with a choice at each element, 2048 x 5120 23 us for 17 of bytes).  The norms' gradients up to 4096 wide:
// a row's work on the vector unit and the sums over it, one after another (2048 x 4096 bf16 29.7 us for 20.3 of bytes).  Wider
// rows: registers.  A lane has two pieces of a row from 4097 elements on and four from 8193 on, and with four (gradients: two) not all of what it holds of
// them stays in registers; the rest lies in scratch memory, up to 0.7 KB for each lane forward and 3.2 KB for the gradients (2048 x 16384 bf16 212 and 1210 us for
// 54 and 81 of bytes, 2048 x 8192 27 and 55 for 27 and 41; floats 467 and 2098 for 108 and 163, 55 and 212 for 54 and 81).
//
// Gradients.  With x^ = (x - mean) r, n = x^ w + b and d the gradient of x^ (d_n w):
//     d_x = r (d - x^ mean(d x^) - mean(d))                 (the last only with a mean)
//     d_w = sum over rows of d_n x^,  d_b = sum over rows of d_n
// mean, r and x^ are made again from the row, which has to be read for x^ anyway: nothing is kept from the forward call.  A workgroup takes rows
// i, i + G, ... (or some of each turn) and keeps the sums over rows of its columns in registers; the G partial sums are added by a second launch,
// in order, so results do not depend on which workgroup ends first.
#include <algorithm>
#include <type_traits>

#include "mmm_elements.h"
#include "mmm_internal.h"

namespace {

constexpr int PIECE = MMM_PIECE;
constexpr int64_t MAX_GROUPS = 1 << 20;   // workgroups of a launch, which may have 2^32 threads: what is left over they take in turns

// The sum over the lanes of a wave, in lane 63: cross-lane moves of the vector unit, sixteen lanes first (a shuffle would go
// through LDS).
template <int CTRL, int ROWS> __device__ __forceinline__ float lanes_below(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xf, true));
}
__device__ __forceinline__ float add_over_lanes(float v)
{
    v += lanes_below<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8
    v += lanes_below<0x112, 0xf>(v);
    v += lanes_below<0x114, 0xf>(v);
    v += lanes_below<0x118, 0xf>(v);
    v += lanes_below<0x142, 0xa>(v);   // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
    v += lanes_below<0x143, 0xc>(v);
    return v;
}

// Sums over a workgroup of at most WAVES waves, the same in every lane.  `room`: not in use by a sum that waves may still be reading (two in turn), zero
// behind the last wave's place.
template <int VALUES, int WAVES> __device__ __forceinline__ void add_over_row(float (&v)[VALUES], float (*room)[WAVES])
{
    typedef float floatx4 __attribute__((ext_vector_type(4)));
    static_assert(WAVES % 4 == 0, "");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int q = 0; q < VALUES; ++q) v[q] = add_over_lanes(v[q]);
    if (lane == 63)
#pragma unroll
        for (int q = 0; q < VALUES; ++q) room[q][wave] = v[q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < VALUES; ++q) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; w += 4) {
            const floatx4 four = *reinterpret_cast<const floatx4 *>(&room[q][w]);
            sum += (four.x + four.y) + (four.z + four.w);
        }
        v[q] = sum;
    }
}
// The same for a workgroup of several rows side by side, WPR waves each: those from wave `first` on.  A row of one wave needs no room, and no barrier.
template <int VALUES, int WPR, int ALL> __device__ __forceinline__ void add_over_rows(float (&v)[VALUES], float (*room)[ALL], int first)
{
    typedef float vec __attribute__((ext_vector_type(WPR < 4 ? 2 : 4)));
    constexpr int PER = WPR < 4 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int q = 0; q < VALUES; ++q) v[q] = add_over_lanes(v[q]);
    if constexpr (WPR == 1) {
#pragma unroll
        for (int q = 0; q < VALUES; ++q) v[q] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[q]), 63));
    } else {
        if (lane == 63)
#pragma unroll
            for (int q = 0; q < VALUES; ++q) room[q][wave] = v[q];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < VALUES; ++q) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WPR; w += PER) {
                const vec some = *reinterpret_cast<const vec *>(&room[q][first + w]);
                if constexpr (PER == 2)
                    sum += some.x + some.y;
                else
                    sum += (some.x + some.y) + (some.z + some.w);
            }
            v[q] = sum;
        }
    }
}
template <int N> __device__ __forceinline__ void clear_rooms(float *rooms)
{
    for (int q = threadIdx.x; q < N; q += blockDim.x) rooms[q] = 0.f;
    __syncthreads();
}

// The pieces of a row that this lane has: V of them, a workgroup's width apart.  Loads are whole pieces that exist, without a branch around any (with
// branches each load was waited for where it stood, and everything under way with it: gradients of 2048 x 4096 bf16 47 us, without 29).
//   EVEN   rows of whole pieces: a lane behind the last one reads that and takes no part (`on`); no choice at each element (29 -> 25 us, 777 x 1992 floats
//          17 -> 15: the row's work on the vector unit is what bounds the gradients)
//   ODD    the last piece begins earlier, at the row's last eight elements, and what of it is another lane's counts for nothing here (`mine`)
//   SHORT  fewer than eight elements: one by one
enum RowKind { EVEN, ODD, SHORT };
template <RowKind KIND, int V> struct Pieces {
    int at[V], first[V], count[V];   // where piece i is read; its elements that are this lane's: first, and how many
    // lane `tid` of the `width` that a row has
    __device__ __forceinline__ Pieces(int N, int tid, int width)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int col = (i * width + tid) * PIECE;
            at[i] = KIND == SHORT ? 0 : min(col, N - PIECE);
            first[i] = KIND == SHORT ? 0 : min(col - at[i], PIECE);
            count[i] = KIND == SHORT ? tid == 0 ? N : 0 : PIECE - first[i];
        }
    }
    __device__ __forceinline__ bool on(int i) const { return KIND != EVEN || first[i] == 0; }
    __device__ __forceinline__ bool mine(int i, int q) const { return KIND == EVEN || (KIND == ODD ? q >= first[i] : q < count[i]); }
    template <typename T> __device__ __forceinline__ typename mmm_raw_piece<T>::type load(const T *row, int i) const
    {
        if constexpr (KIND != SHORT) {
            typedef typename mmm_row_piece<T, PIECE>::type piece;
            return *reinterpret_cast<const piece *>(row + at[i]);
        } else {
            return mmm_load_raw(row, count[i]);
        }
    }
    // (where the piece is on)
    template <typename T> __device__ __forceinline__ void store(T *row, int i, const float (&v)[PIECE]) const
    {
        if (KIND == EVEN || (KIND == ODD && first[i] == 0)) {
            mmm_store_piece(row + at[i], PIECE, v);
        } else {
#pragma unroll
            for (int q = 0; q < PIECE; ++q)
                if (mine(i, q)) row[at[i] + q] = (T)v[q];
        }
    }
};

// Operands that are not there are given an address that may be read all the same, and a flag: what is read there is replaced.
struct NormParams {
    mmm_block_norm_desc d;
    float inv_n;
    const void *h, *y, *gate, *post_weight, *post_bias, *pre_weight, *pre_bias;
    int64_t ldh, ldy, ldgate;
    void *h_out, *n;
    int64_t ldh_out, ldn;
    const void *row_gates;   // MMM_GATE_ROW: the values
    bool has_y, has_gate, has_post_weight, has_post_bias, has_pre_weight, has_pre_bias;   // has_gate: a value per column or element
};

// values of a piece, or one and the same where there are none
template <typename R> __device__ __forceinline__ void values_or(const R &raw, bool there, float otherwise, float (&out)[PIECE])
{
#pragma unroll
    for (int q = 0; q < PIECE; ++q) out[q] = there ? (float)raw[q] : otherwise;
}

template <typename T, typename TH, typename TY, int V, int WAVES, RowKind KIND> __global__ __launch_bounds__(64 * WAVES) void mmm_block_norm_kernel(const NormParams p)
{
    __shared__ __align__(16) float rooms[2][4][1][WAVES];   // (rows in turn: of a row, a wave may still read what another has gone past)
    clear_rooms<2 * 4 * WAVES>(&rooms[0][0][0][0]);
    const Pieces<KIND, V> mine((int)p.d.N, (int)threadIdx.x, (int)blockDim.x);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.d.M; row += gridDim.x, turn ^= 1) {
        float h[V][PIECE], v[V][PIECE];
        typename mmm_raw_piece<TH>::type raw_h[V];
        typename mmm_raw_piece<TY>::type raw_y[V];
        typename mmm_raw_piece<T>::type raw_gate[V], raw_w[V], raw_b[V], raw_w2[V], raw_b2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            raw_h[i] = mine.load(static_cast<const TH *>(p.h) + row * p.ldh, i);
            raw_y[i] = mine.load(static_cast<const TY *>(p.y) + row * p.ldy, i);
            raw_gate[i] = mine.load(static_cast<const T *>(p.gate) + row * p.ldgate, i);
            raw_w[i] = mine.load(static_cast<const T *>(p.post_weight), i);
            raw_b[i] = mine.load(static_cast<const T *>(p.post_bias), i);
            raw_w2[i] = mine.load(static_cast<const T *>(p.pre_weight), i);
            raw_b2[i] = mine.load(static_cast<const T *>(p.pre_bias), i);
        }
        // 1 / the deviation of the row in x, whose mean is taken off it; `of`: which of the two norms
        auto standard = [&](float (&x)[V][PIECE], int32_t kind, int of) __attribute__((always_inline)) -> float {
            float sum[1] = {0.f};
            if (kind == MMM_NORM_LAYER) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (mine.on(i))
#pragma unroll
                        for (int q = 0; q < PIECE; ++q) sum[0] += x[i][q];   // (elements that are not this lane's are zero)
                add_over_row(sum, rooms[turn][of]);
                const float mean = sum[0] * p.inv_n;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (mine.on(i))
#pragma unroll
                        for (int q = 0; q < PIECE; ++q) x[i][q] = mine.mine(i, q) ? x[i][q] - mean : 0.f;
                sum[0] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (mine.on(i))
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) sum[0] += x[i][q] * x[i][q];
            add_over_row(sum, rooms[turn][2 + of]);
            return 1.f / sqrtf(sum[0] * p.inv_n + p.d.eps);
        };
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (mine.on(i))
#pragma unroll
                for (int q = 0; q < PIECE; ++q) {
                    h[i][q] = mine.mine(i, q) ? (float)raw_h[i][q] : 0.f;
                    v[i][q] = mine.mine(i, q) ? (float)raw_y[i][q] : 0.f;
                }
        if (p.has_y) {
            const float r = p.d.post != MMM_NORM_NONE ? standard(v, p.d.post, 0) : 1.f;
            const float row_gate = p.d.gate == MMM_GATE_ROW ? (float)static_cast<const T *>(p.row_gates)[row] : 1.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!mine.on(i)) continue;
                float w[PIECE], b[PIECE], g[PIECE];
                values_or(raw_w[i], p.has_post_weight, 1.f, w);
                values_or(raw_b[i], p.has_post_bias, 0.f, b);
                values_or(raw_gate[i], p.has_gate, row_gate, g);
#pragma unroll
                for (int q = 0; q < PIECE; ++q) h[i][q] = mine.mine(i, q) ? p.d.alpha * h[i][q] + g[q] * (v[i][q] * r * w[q] + b[q]) : 0.f;
                if (p.h_out != nullptr) mine.store(static_cast<TH *>(p.h_out) + row * p.ldh_out, i, h[i]);
            }
        }
        if (p.d.pre != MMM_NORM_NONE) {
            const float r = standard(h, p.d.pre, 1);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!mine.on(i)) continue;
                float w[PIECE], b[PIECE];
                values_or(raw_w2[i], p.has_pre_weight, 1.f, w);
                values_or(raw_b2[i], p.has_pre_bias, 0.f, b);
#pragma unroll
                for (int q = 0; q < PIECE; ++q) h[i][q] = h[i][q] * r * w[q] + b[q];
                mine.store(static_cast<T *>(p.n) + row * p.ldn, i, h[i]);
            }
        }
    }
}

// sums over rows, in this order in the workspace
enum { SUM_PRE_WEIGHT, SUM_PRE_BIAS, SUM_POST_WEIGHT, SUM_POST_BIAS, SUM_GATE, SUMS };

struct NormGradParams {
    mmm_block_norm_desc d;
    mmm_block_norm_grads g;   // (operands that are not there: as above)
    float inv_n;
    float *partials;        // [workgroup][sum asked for][N]
    int32_t place[SUMS];    // of a sum among those asked for; -1: not asked for
    int32_t sums;
    const void *row_gates;
    bool has_d_h_out, has_gate, has_post_weight, has_post_bias, has_pre_weight, block;
};

// What a row takes from memory: asked for while the row before is worked on.
template <typename T, typename TH, typename TY, int V, RowKind KIND> struct GradRow {
    typename mmm_raw_piece<TH>::type x[V], d[V];
    typename mmm_raw_piece<T>::type dn[V], gate[V];
    typename mmm_raw_piece<TY>::type y[V];
    __device__ __forceinline__ void load(const NormGradParams &p, const Pieces<KIND, V> &mine, int64_t row)
    {
        const mmm_block_norm_grads &g = p.g;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = mine.load(static_cast<const TH *>(g.h_out) + row * g.ldh_out, i);
            dn[i] = mine.load(static_cast<const T *>(g.d_n) + row * g.ldd_n, i);
            d[i] = mine.load(static_cast<const TH *>(g.d_h_out) + row * g.ldd_h_out, i);
            y[i] = mine.load(static_cast<const TY *>(g.y) + row * g.ldy, i);
            gate[i] = mine.load(static_cast<const T *>(g.gate_values) + row * g.ldgate, i);
        }
    }
};
// What all rows share.
template <typename T, int V, RowKind KIND> struct GradColumns {
    typename mmm_raw_piece<T>::type pre_weight[V], post_weight[V], post_bias[V];
    __device__ __forceinline__ void load(const NormGradParams &p, const Pieces<KIND, V> &mine, bool biases)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            typedef typename mmm_raw_piece<T>::type raw;
            pre_weight[i] = mine.load(static_cast<const T *>(p.g.pre_weight), i);
            post_weight[i] = mine.load(static_cast<const T *>(p.g.post_weight), i);
            if (biases) post_bias[i] = mine.load(static_cast<const T *>(p.g.post_bias), i);
            if (!p.has_pre_weight) pre_weight[i] = raw((T)1.f);
            if (!p.has_post_weight) post_weight[i] = raw((T)1.f);
            if (!biases || !p.has_post_bias) post_bias[i] = raw((T)0.f);
        }
    }
};

// Rows side by side in a workgroup, of WPR waves each
constexpr int rows_beside(int wpr) { return wpr >= 8 ? 1 : 8 / wpr; }
// BIASES: the norm behind the block has a bias, or sums for biases are asked for
template <typename T, typename TH, typename TY, int V, int WPR, bool BIASES, RowKind KIND>
__global__ __launch_bounds__(64 * WPR * rows_beside(WPR)) void mmm_block_norm_grad_kernel(const NormGradParams p)
{
    constexpr int SIDE = rows_beside(WPR), WAVES = WPR * SIDE;
    __shared__ __align__(16) float rooms[2][4][3][WAVES];   // (rows in turn, as above)
    __shared__ float fold[SIDE > 1 ? SIDE - 1 : 1][SIDE > 1 ? V * PIECE : 1][64 * WPR];
    clear_rooms<2 * 4 * 3 * WAVES>(&rooms[0][0][0][0]);
    const mmm_block_norm_grads &g = p.g;
    const int beside = SIDE > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / (64 * WPR)) : 0, first = beside * WPR;   // which of the rows side by side
    const int tid = (int)threadIdx.x - beside * 64 * WPR;
    const Pieces<KIND, V> mine((int)p.d.N, tid, SIDE > 1 ? 64 * WPR : (int)blockDim.x);
    const bool pre = p.d.pre != MMM_NORM_NONE, block = p.block, post = p.d.post != MMM_NORM_NONE;
    const bool pre_mean = p.d.pre == MMM_NORM_LAYER, post_mean = p.d.post == MMM_NORM_LAYER;
    float sums[SUMS][V][PIECE];
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int q = 0; q < PIECE; ++q) sums[s][i][q] = 0.f;

    GradColumns<T, V, KIND> columns;
    if (V == 1) columns.load(p, mine, BIASES);   // (wider rows have no registers for them)
    GradRow<T, TH, TY, V, KIND> next;
    next.load(p, mine, min((int64_t)blockIdx.x * SIDE + beside, p.d.M - 1));
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * SIDE; row0 < p.d.M; row0 += (int64_t)gridDim.x * SIDE, turn ^= 1) {
        // (behind the last row: that one again, with gradients of zero, and nothing is stored)
        const bool there = SIDE == 1 || row0 + beside < p.d.M;
        const int64_t row = there ? row0 + beside : p.d.M - 1;
        float x[V][PIECE], dn[V][PIECE], d[V][PIECE], y[V][PIECE], gate[V][PIECE];
        const float row_gate = p.d.gate == MMM_GATE_ROW ? (float)static_cast<const T *>(p.row_gates)[row] : 1.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!mine.on(i)) continue;
            values_or(next.gate[i], p.has_gate, row_gate, gate[i]);
#pragma unroll
            for (int q = 0; q < PIECE; ++q) {   // (zeros for what is another lane's; of operands that are not there nothing is used)
                const bool on = mine.mine(i, q);
                x[i][q] = on ? (float)next.x[i][q] : 0.f;
                dn[i][q] = on && there ? (float)next.dn[i][q] : 0.f;
                d[i][q] = p.has_d_h_out && on && there ? (float)next.d[i][q] : 0.f;
                y[i][q] = on ? (float)next.y[i][q] : 0.f;
            }
        }
        if (V > 1) columns.load(p, mine, BIASES);
        next.load(p, mine, min(row0 + (int64_t)gridDim.x * SIDE + beside, p.d.M - 1));
        // both rows standardised together: one sum for means, one for variances
        float s2[2] = {0.f, 0.f};
        if (pre_mean || post_mean) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (mine.on(i))
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) {
                        s2[0] += x[i][q];
                        s2[1] += y[i][q];
                    }
            add_over_rows<sizeof(s2) / sizeof(float), WPR, WAVES>(s2, rooms[turn][0], first);
            const float mx = pre_mean ? s2[0] * p.inv_n : 0.f, my = post_mean ? s2[1] * p.inv_n : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (mine.on(i))
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) {
                        x[i][q] = mine.mine(i, q) ? x[i][q] - mx : 0.f;
                        y[i][q] = mine.mine(i, q) ? y[i][q] - my : 0.f;
                    }
            s2[0] = s2[1] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (mine.on(i))
#pragma unroll
                for (int q = 0; q < PIECE; ++q) {
                    s2[0] += x[i][q] * x[i][q];
                    s2[1] += y[i][q] * y[i][q];
                }
        add_over_rows<sizeof(s2) / sizeof(float), WPR, WAVES>(s2, rooms[turn][1], first);
        const float rx = 1.f / sqrtf(s2[0] * p.inv_n + p.d.eps), ry = post ? 1.f / sqrtf(s2[1] * p.inv_n + p.d.eps) : 1.f;
        // through the norm in front of the next block: d becomes the gradient of h'
        if (pre) {
            float c[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!mine.on(i)) continue;
#pragma unroll
                for (int q = 0; q < PIECE; ++q) {
                    x[i][q] *= rx;
                    sums[SUM_PRE_WEIGHT][i][q] += dn[i][q] * x[i][q];
                    if (BIASES) sums[SUM_PRE_BIAS][i][q] += dn[i][q];
                    dn[i][q] *= (float)columns.pre_weight[i][q];
                    c[0] += dn[i][q] * x[i][q];
                    c[1] += dn[i][q];
                }
            }
            add_over_rows<sizeof(c) / sizeof(float), WPR, WAVES>(c, rooms[turn][2], first);
            const float along = c[0] * p.inv_n, mean = pre_mean ? c[1] * p.inv_n : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (mine.on(i))
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) d[i][q] += rx * (dn[i][q] - x[i][q] * along - mean);
        }
        if (g.d_h != nullptr && there) {
            const float alpha = block ? p.d.alpha : 1.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!mine.on(i)) continue;
                float out[PIECE];
#pragma unroll
                for (int q = 0; q < PIECE; ++q) out[q] = alpha * d[i][q];
                mine.store(static_cast<TH *>(g.d_h) + row * g.ldd_h, i, out);
            }
        }
        if (!block) continue;   // (uniform: no sum is under way)
        // through gate and norm behind the block: d becomes the gradient of y
        float c[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!mine.on(i)) continue;
            float dgate[PIECE];
#pragma unroll
            for (int q = 0; q < PIECE; ++q) {
                if (!mine.mine(i, q)) d[i][q] = 0.f;   // (the mean has been taken off there, too)
                y[i][q] *= ry;
                const float w = (float)columns.post_weight[i][q];
                dgate[q] = d[i][q] * (BIASES ? y[i][q] * w + (float)columns.post_bias[i][q] : y[i][q] * w);
                c[2] += dgate[q];
                sums[SUM_GATE][i][q] += dgate[q];
                d[i][q] *= gate[i][q];
                sums[SUM_POST_WEIGHT][i][q] += d[i][q] * y[i][q];
                if (BIASES) sums[SUM_POST_BIAS][i][q] += d[i][q];
                d[i][q] *= w;
                c[0] += d[i][q] * y[i][q];
                c[1] += d[i][q];
            }
            if (p.d.gate == MMM_GATE_FULL && g.d_gate != nullptr && there) mine.store(static_cast<T *>(g.d_gate) + row * g.ldd_gate, i, dgate);
        }
        add_over_rows<sizeof(c) / sizeof(float), WPR, WAVES>(c, rooms[turn][3], first);
        if (p.d.gate == MMM_GATE_ROW && g.d_gate != nullptr && there && tid == 0) static_cast<float *>(g.d_gate)[row] = c[2];
        if (g.d_y != nullptr && there) {
            const float along = post ? c[0] * p.inv_n : 0.f, mean = post_mean ? c[1] * p.inv_n : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!mine.on(i)) continue;
#pragma unroll
                for (int q = 0; q < PIECE; ++q) d[i][q] = ry * (d[i][q] - y[i][q] * along - mean);
                mine.store(static_cast<TY *>(g.d_y) + row * g.ldd_y, i, d[i]);
            }
        }
    }
    if (p.sums == 0) return;
#pragma unroll
    for (int s = 0; s < SUMS; ++s) {
        if (p.place[s] < 0) continue;
        if constexpr (SIDE > 1) {   // the rows side by side, in order
            __syncthreads();
            if (beside > 0)
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) fold[beside - 1][i * PIECE + q][tid] = sums[s][i][q];
            __syncthreads();
            if (beside > 0) continue;
#pragma unroll
            for (int b = 0; b < SIDE - 1; ++b)
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) sums[s][i][q] += fold[b][i * PIECE + q][tid];
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (mine.on(i)) mine.store(p.partials + ((int64_t)blockIdx.x * p.sums + p.place[s]) * p.d.N, i, sums[s][i]);
    }
}

// Gradient through the epilogue.  A wave owns 512 neighbouring columns and every fourth row of its workgroup's share of them.
struct ActParams {
    const void *dC, *Z;
    void *dZ;
    int64_t lddc, ldz, lddz, M, N;
    int64_t rows;       // per workgroup
    int32_t activation;
    float *partials;    // [share of rows][N]; null: no sums asked for
};
constexpr int ACT_COLS = 64 * PIECE, ACT_WAVES = 4;

template <typename T, typename TC> __global__ __launch_bounds__(64 * ACT_WAVES) void mmm_epilogue_grad_kernel(const ActParams p)
{
    __shared__ float room[ACT_WAVES][ACT_COLS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * ACT_COLS + lane * PIECE;
    const int left = (int)min((int64_t)PIECE, p.N - col);
    const int64_t end = min(p.M, ((int64_t)blockIdx.y + 1) * p.rows);
    float sum[PIECE] = {};
    if (left > 0) {
        for (int64_t row = (int64_t)blockIdx.y * p.rows + wave; row < end; row += ACT_WAVES) {
            float d[PIECE], z[PIECE];
            mmm_load_piece(static_cast<const TC *>(p.dC) + row * p.lddc + col, left, d);
            if (p.activation != MMM_ACT_NONE) {
                mmm_load_piece(static_cast<const TC *>(p.Z) + row * p.ldz + col, left, z);
                mmm_apply_slope<T>(d, z, p.activation);
            }
#pragma unroll
            for (int q = 0; q < PIECE; ++q) sum[q] += d[q];
            if (p.dZ != nullptr) mmm_store_piece(static_cast<T *>(p.dZ) + row * p.lddz + col, left, d);
        }
    }
    if (p.partials == nullptr) return;
#pragma unroll
    for (int q = 0; q < PIECE; ++q) room[wave][lane * PIECE + q] = sum[q];
    __syncthreads();
    for (int c = threadIdx.x; c < ACT_COLS; c += 64 * ACT_WAVES) {
        const int64_t at = (int64_t)blockIdx.x * ACT_COLS + c;
        float s = room[0][c];
        for (int w = 1; w < ACT_WAVES; ++w) s += room[w][c];
        if (at < p.N) p.partials[(int64_t)blockIdx.y * p.N + at] = s;
    }
}

// Partial sums added in order: out[s][j] = sum over g of partials[g][s][j].  A wave takes every sixteenth g of 64 columns, eight of them in flight.
struct ReduceParams {
    const float *partials;
    int64_t groups, N;
    int32_t sums;
    float *out[SUMS];
};
constexpr int REDUCE_WAVES = 16;

__global__ __launch_bounds__(64 * REDUCE_WAVES) void mmm_add_partials_kernel(const ReduceParams p)
{
    __shared__ float room[REDUCE_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int s = (int)blockIdx.y;
    float *out = p.out[0];
#pragma unroll
    for (int q = 1; q < SUMS; ++q)
        if (q == s) out = p.out[q];
    for (int64_t col0 = (int64_t)blockIdx.x * 64; col0 < p.N; col0 += (int64_t)gridDim.x * 64) {
        const int64_t col = min(col0 + lane, p.N - 1), step = (int64_t)p.sums * p.N;
        const float *const at = p.partials + (int64_t)s * p.N + col;
        float sum = 0.f;
        for (int64_t g = wave; g < p.groups; g += 8 * REDUCE_WAVES) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = at[min(g + i * REDUCE_WAVES, p.groups - 1) * step];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += g + i * REDUCE_WAVES < p.groups ? v[i] : 0.f;
        }
        room[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && col0 + lane < p.N) {
            for (int w = 1; w < REDUCE_WAVES; ++w) sum += room[w][lane];
            out[col] = sum;
        }
        __syncthreads();   // (read before the next columns are written)
    }
}

hipError_t add_partials(const ReduceParams &r, hipStream_t s)
{
    hipLaunchKernelGGL(mmm_add_partials_kernel, dim3((uint32_t)std::min<int64_t>((r.N + 63) / 64, MAX_GROUPS), (uint32_t)r.sums), dim3(64 * REDUCE_WAVES), 0, s, r);
    return hipGetLastError();
}

// Threads and pieces per lane for a row: one piece as long as the workgroup has room.
struct RowShape { uint32_t threads; int pieces; };
RowShape row_shape(int64_t N)
{
    const uint32_t lanes = (uint32_t)((N + PIECE - 1) / PIECE);
    const int pieces = lanes <= 512 ? 1 : lanes <= 1024 ? 2 : 4;
    return {((lanes + (uint32_t)pieces - 1) / (uint32_t)pieces + 63) / 64 * 64, pieces};
}

// calls f with the types of a case
template <typename T, typename F> auto with_stream_types(const mmm_block_norm_desc &d, F f)
{
    if constexpr (std::is_same_v<T, float>) {
        return f(T{}, T{}, T{});
    } else {
        if (d.dt_h == MMM_F32) return d.dt_y == MMM_F32 ? f(T{}, float{}, float{}) : f(T{}, float{}, T{});
        return d.dt_y == MMM_F32 ? f(T{}, T{}, float{}) : f(T{}, T{}, T{});
    }
}
template <typename F> auto with_types(const mmm_block_norm_desc &d, F f)
{
    if (d.dt == MMM_BF16) return with_stream_types<__bf16>(d, f);
    if (d.dt == MMM_F16) return with_stream_types<_Float16>(d, f);
    return with_stream_types<float>(d, f);
}

// Waves for a row of the gradients, and pieces per lane.  Rows of whole pieces of up to 2048 elements stand side by side in a workgroup of eight waves (2, 4 or 8): they share
// its barriers, a row of one wave needs none, and partial sums are fewer (2048 x 512 half beside float, with biases, 29 -> 12 us; 8192 x 1024 bf16 32 -> 26;
// 777 x 1992 floats 19.8 -> 18.1; 4096 wide in two pieces per lane, two rows beside each other, has no registers for the columns: 29 -> 31).
struct GradShape { uint32_t threads; int pieces, waves, beside; };
GradShape grad_shape(int64_t N)
{
    const RowShape r = row_shape(N);
    if (N >= PIECE && (N % PIECE != 0 || N > 2048)) return {r.threads, r.pieces, r.pieces == 4 ? 16 : 8, 1};
    const int waves = N <= 512 ? 1 : N <= 1024 ? 2 : 4;
    return {512, 1, waves, rows_beside(waves)};
}
// Workgroups of the gradients: as many as the registers of the chip hold at a time (8 waves on a compute unit), so that partial sums are few, and
// all with the same number of turns but for one.  2048 x 4096 bf16, an older form: 256 groups 28.6 us and 4.0 for adding up, 512 32.3 and 5.5, 1024 38.8 and 8.3.
int64_t norm_grad_groups(int64_t M, int64_t N)
{
    const GradShape shape = grad_shape(N);
    const int64_t slots = 256 * (shape.beside > 1 ? 1 : std::max<int64_t>(1, 512 / shape.threads)), turns = (M + shape.beside - 1) / shape.beside, each = (turns + slots - 1) / slots;
    return (turns + each - 1) / each;
}
int64_t act_strips(int64_t N) { return (N + ACT_COLS - 1) / ACT_COLS; }
int64_t act_shares(int64_t M, int64_t N)
{
    return std::min<int64_t>((M + ACT_WAVES - 1) / ACT_WAVES, std::max<int64_t>(1, 2048 / act_strips(N)));
}

}   // namespace

hipError_t mmm_launch_block_norm(const mmm_block_norm_desc &d, const void *h, int64_t ldh, const void *y, int64_t ldy, const void *gate, int64_t ldgate,
                                 const void *post_weight, const void *post_bias, const void *pre_weight, const void *pre_bias, void *h_out,
                                 int64_t ldh_out, void *n, int64_t ldn, hipStream_t s)
{
    if (d.M < 1 || d.N < 1 || d.N > MMM_NORM_MAX_WIDTH) return hipErrorInvalidValue;
    const RowShape shape = row_shape(d.N);
    NormParams p{d, 1.f / (float)d.N, h, y, gate, post_weight, post_bias, pre_weight, pre_bias, ldh, ldy, ldgate, h_out, n, ldh_out, ldn,
                 gate, y != nullptr, d.gate >= MMM_GATE_COL, post_weight != nullptr, post_bias != nullptr, pre_weight != nullptr, pre_bias != nullptr};
    // what is not there is read from h, whose rows are N elements of no smaller a type (without a block y has that type, too)
    if (y == nullptr) {
        p.y = h;
        p.ldy = ldh;
        p.d.dt_y = d.dt_h;
    }
    if (d.gate < MMM_GATE_FULL) p.ldgate = 0;
    if (!p.has_gate) p.gate = h;
    for (const void **q : {&p.post_weight, &p.post_bias, &p.pre_weight, &p.pre_bias})
        if (*q == nullptr) *q = h;
    (void)hipGetLastError();
    with_types(p.d, [&](auto t, auto th, auto ty) {
        typedef decltype(t) T;
        typedef decltype(th) TH;
        typedef decltype(ty) TY;
        void (*fn)(const NormParams) = d.N < PIECE              ? mmm_block_norm_kernel<T, TH, TY, 1, 4, SHORT>
                                       : shape.pieces == 2      ? mmm_block_norm_kernel<T, TH, TY, 2, 8, ODD>
                                       : shape.pieces == 4      ? mmm_block_norm_kernel<T, TH, TY, 4, 16, ODD>
                                       : d.N % PIECE != 0       ? mmm_block_norm_kernel<T, TH, TY, 1, 8, ODD>
                                       : shape.threads <= 256   ? mmm_block_norm_kernel<T, TH, TY, 1, 4, EVEN>
                                                                : mmm_block_norm_kernel<T, TH, TY, 1, 8, EVEN>;
        hipLaunchKernelGGL(fn, dim3((uint32_t)std::min(d.M, MAX_GROUPS)), dim3(shape.threads), 0, s, p);
        return 0;
    });
    return hipGetLastError();
}

size_t mmm_block_norm_grad_bytes(int64_t M, int64_t N) { return (size_t)norm_grad_groups(M, N) * (size_t)N * SUMS * sizeof(float); }

hipError_t mmm_launch_block_norm_grad(const mmm_block_norm_desc &d, const mmm_block_norm_grads &g, void *workspace, hipStream_t s)
{
    if (d.M < 1 || d.N < 1 || d.N > MMM_NORM_MAX_WIDTH) return hipErrorInvalidValue;
    const GradShape shape = grad_shape(d.N);
    NormGradParams p{d, g, 1.f / (float)d.N, static_cast<float *>(workspace), {}, 0, g.gate_values, g.d_h_out != nullptr, d.gate >= MMM_GATE_COL, g.post_weight != nullptr,
                     g.post_bias != nullptr, g.pre_weight != nullptr, g.y != nullptr};
    // What is not there is read from what is: h' and d_n with a norm in front, else d_h' and y (the types of a block that is not there are
    // those of h, and the rows of a narrower type end sooner).
    const bool pre = d.pre != MMM_NORM_NONE;
    if (!pre) {
        p.g.h_out = p.g.d_n = g.d_h_out;
        p.g.ldh_out = p.g.ldd_n = g.ldd_h_out;
    }
    if (g.d_h_out == nullptr) {
        p.g.d_h_out = g.h_out;
        p.g.ldd_h_out = g.ldh_out;
    }
    if (g.y == nullptr) {
        p.g.y = p.g.h_out;
        p.g.ldy = p.g.ldh_out;
        p.d.dt_y = d.dt_h;
    }
    if (d.gate < MMM_GATE_FULL) p.g.ldgate = 0;
    if (!p.has_gate) p.g.gate_values = p.g.h_out;
    for (const void **q : {&p.g.post_weight, &p.g.post_bias, &p.g.pre_weight})
        if (*q == nullptr) *q = p.g.h_out;
    float *const out[SUMS] = {g.d_pre_weight, g.d_pre_bias, g.d_post_weight, g.d_post_bias, d.gate == MMM_GATE_COL ? static_cast<float *>(g.d_gate) : nullptr};
    const int64_t groups = norm_grad_groups(d.M, d.N);
    ReduceParams r{p.partials, groups, d.N, 0, {}};
    for (int q = 0; q < SUMS; ++q) {
        p.place[q] = out[q] != nullptr ? r.sums : -1;
        if (out[q] != nullptr) r.out[r.sums++] = out[q];
    }
    p.sums = r.sums;
    (void)hipGetLastError();
    with_types(p.d, [&](auto t, auto th, auto ty) {
        typedef decltype(t) T;
        typedef decltype(th) TH;
        typedef decltype(ty) TY;
        const bool biases = g.d_pre_bias != nullptr || g.d_post_bias != nullptr || g.post_bias != nullptr;
        void (*fn)(const NormGradParams);
        if (d.N < PIECE)
            fn = mmm_block_norm_grad_kernel<T, TH, TY, 1, 1, true, SHORT>;
        else if (shape.pieces == 4)
            fn = mmm_block_norm_grad_kernel<T, TH, TY, 4, 16, true, ODD>;
        else if (shape.pieces == 2)
            fn = mmm_block_norm_grad_kernel<T, TH, TY, 2, 8, true, ODD>;
        else if (d.N % PIECE != 0)
            fn = mmm_block_norm_grad_kernel<T, TH, TY, 1, 8, true, ODD>;
        else if (shape.waves == 1)
            fn = biases ? mmm_block_norm_grad_kernel<T, TH, TY, 1, 1, true, EVEN> : mmm_block_norm_grad_kernel<T, TH, TY, 1, 1, false, EVEN>;
        else if (shape.waves == 2)
            fn = biases ? mmm_block_norm_grad_kernel<T, TH, TY, 1, 2, true, EVEN> : mmm_block_norm_grad_kernel<T, TH, TY, 1, 2, false, EVEN>;
        else if (shape.waves == 4)
            fn = biases ? mmm_block_norm_grad_kernel<T, TH, TY, 1, 4, true, EVEN> : mmm_block_norm_grad_kernel<T, TH, TY, 1, 4, false, EVEN>;
        else
            fn = biases ? mmm_block_norm_grad_kernel<T, TH, TY, 1, 8, true, EVEN> : mmm_block_norm_grad_kernel<T, TH, TY, 1, 8, false, EVEN>;
        hipLaunchKernelGGL(fn, dim3((uint32_t)groups), dim3(shape.threads), 0, s, p);
        return 0;
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || r.sums == 0) return e;
    return add_partials(r, s);
}

size_t mmm_epilogue_grad_bytes(int64_t M, int64_t N) { return (size_t)act_shares(M, N) * (size_t)N * sizeof(float); }

hipError_t mmm_launch_epilogue_grad(int64_t M, int64_t N, int32_t dt, int32_t out_dtype, int32_t activation, const void *dC, int64_t lddc, const void *Z,
                                    int64_t ldz, void *dZ, int64_t lddz, float *dbias, void *workspace, hipStream_t s)
{
    const int64_t strips = act_strips(N), shares = act_shares(M, N);
    if (M < 1 || N < 1 || strips > 0x7fffffffLL || shares > 65535) return hipErrorInvalidValue;
    const ActParams p{dC, Z, dZ, lddc, ldz, lddz, M, N, (M + shares - 1) / shares, activation, dbias != nullptr ? static_cast<float *>(workspace) : nullptr};
    void (*fn)(const ActParams);
    if (dt == MMM_F32)
        fn = mmm_epilogue_grad_kernel<float, float>;
    else if (dt == MMM_BF16)
        fn = out_dtype == MMM_F32 ? mmm_epilogue_grad_kernel<__bf16, float> : mmm_epilogue_grad_kernel<__bf16, __bf16>;
    else
        fn = out_dtype == MMM_F32 ? mmm_epilogue_grad_kernel<_Float16, float> : mmm_epilogue_grad_kernel<_Float16, _Float16>;
    (void)hipGetLastError();
    hipLaunchKernelGGL(fn, dim3((uint32_t)strips, (uint32_t)shares), dim3(64 * ACT_WAVES), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || dbias == nullptr) return e;
    ReduceParams r{static_cast<const float *>(workspace), shares, N, 1, {dbias}};
    return add_partials(r, s);
}
