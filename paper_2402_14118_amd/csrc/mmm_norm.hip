// The norms around a block with its gate and residual (mmm_block_norm), their gradients, and the gradient through the epilogue of
// the multiplication: the operators of a residual block that touch every element a few times.
//
//     v = norm_post(y) w + b        h' = alpha h + g v        n = norm_pre(h') w' + b'
//
// All are bound by HBM, so each reads its inputs and writes its outputs once.  A workgroup keeps a row in registers, eight neighbours (16 bytes of
// a 16-bit type) per lane and piece; both norms, gate and residual work on that.  Sums of a row: lanes by shuffles, waves through LDS, in a
// fixed order.  The variance is that of the centred row, which stands in registers anyway, not a difference of two sums.
//
// Gradients.  With x^ = (x - mean) r, n = x^ w + b and d the gradient of x^ (d_n w):
//     d_x = r (d - x^ mean(d x^) - mean(d))                 (the last only with a mean)
//     d_w = sum over rows of d_n x^,  d_b = sum over rows of d_n
// mean, r and x^ are made again from the row, which has to be read for x^ anyway: nothing is kept from the forward call.  A workgroup takes rows
// i, i + G, ... and keeps the sums over rows of its columns in registers; the G partial sums are added by a second launch,
// in order, so results do not depend on which workgroup ends first.
#include <algorithm>
#include <type_traits>

#include "mmm_elements.h"
#include "mmm_internal.h"

namespace {

constexpr int PIECE = MMM_PIECE;
constexpr int64_t MAX_GROUPS = 1 << 20;   // workgroups of a launch, which may have 2^32 threads: what is left over they take in turns

template <int VALUES> __device__ __forceinline__ void add_over_lanes(float (&v)[VALUES])
{
#pragma unroll
    for (int step = 1; step < 64; step *= 2)
#pragma unroll
        for (int q = 0; q < VALUES; ++q) v[q] += __shfl_xor(v[q], step, 64);
}

// Sums over a workgroup, the same in every lane.  `room`: VALUES floats per wave, not in use by a sum that waves may still be reading (two in turn).
template <int VALUES> __device__ __forceinline__ void add_over_row(float (&v)[VALUES], float *room, int waves)
{
    add_over_lanes(v);
    if (waves == 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0)
#pragma unroll
        for (int q = 0; q < VALUES; ++q) room[wave * VALUES + q] = v[q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < VALUES; ++q) {
        float sum = room[q];
        for (int w = 1; w < waves; ++w) sum += room[w * VALUES + q];
        v[q] = sum;
    }
}

struct NormParams {
    mmm_block_norm_desc d;
    float inv_n;
    const void *h, *y, *gate, *post_weight, *post_bias, *pre_weight, *pre_bias;
    int64_t ldh, ldy, ldgate;
    void *h_out, *n;
    int64_t ldh_out, ldn;
};

// the pieces of a row that this lane has: V of them, a workgroup's width apart
#define MMM_FOR_PIECES(p, col, left)                                                                              \
    _Pragma("unroll") for (int p = 0; p < V; ++p)                                                                 \
        if (const int col = (p * (int)blockDim.x + (int)threadIdx.x) * PIECE, left = N - col; left > 0)

template <typename T, typename TH, typename TY, int V> __global__ __launch_bounds__(1024) void mmm_block_norm_kernel(const NormParams p)
{
    __shared__ float rooms[2][4][16];   // (rows in turn: of a row, a wave may still read what another has gone past)
    const int N = (int)p.d.N, waves = (int)blockDim.x >> 6;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.d.M; row += gridDim.x, turn ^= 1) {
        float h[V][PIECE], v[V][PIECE];
        MMM_FOR_PIECES(i, col, left) mmm_load_piece(static_cast<const TH *>(p.h) + row * p.ldh + col, left, h[i]);
        // 1 / the deviation of the row in x, whose mean is taken off it; `of`: which of the two norms
        auto standard = [&](float (&x)[V][PIECE], int32_t kind, int of) __attribute__((always_inline)) -> float {
            float sum[1] = {0.f};
            if (kind == MMM_NORM_LAYER) {
                MMM_FOR_PIECES(i, col, left)
                {
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) sum[0] += x[i][q];   // (elements past the row are zero)
                }
                add_over_row(sum, rooms[turn][of], waves);
                const float mean = sum[0] * p.inv_n;
                MMM_FOR_PIECES(i, col, left)
                {
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) x[i][q] = q < left ? x[i][q] - mean : 0.f;
                }
                sum[0] = 0.f;
            }
            MMM_FOR_PIECES(i, col, left)
            {
#pragma unroll
                for (int q = 0; q < PIECE; ++q) sum[0] += x[i][q] * x[i][q];
            }
            add_over_row(sum, rooms[turn][2 + of], waves);
            return 1.f / sqrtf(sum[0] * p.inv_n + p.d.eps);
        };
        auto affine = [&](float (&x)[PIECE], float r, const void *weight, const void *bias, int col, int left) __attribute__((always_inline)) {
            float w[PIECE], b[PIECE];
            if (weight != nullptr) mmm_load_piece(static_cast<const T *>(weight) + col, left, w);
            if (bias != nullptr) mmm_load_piece(static_cast<const T *>(bias) + col, left, b);
#pragma unroll
            for (int q = 0; q < PIECE; ++q) {
                x[q] *= r;
                if (weight != nullptr) x[q] *= w[q];
                if (bias != nullptr) x[q] += b[q];
            }
        };
        if (p.y != nullptr) {
            MMM_FOR_PIECES(i, col, left) mmm_load_piece(static_cast<const TY *>(p.y) + row * p.ldy + col, left, v[i]);
            const float r = p.d.post != MMM_NORM_NONE ? standard(v, p.d.post, 0) : 1.f;
            const float row_gate = p.d.gate == MMM_GATE_ROW ? (float)static_cast<const T *>(p.gate)[row] : 1.f;
            MMM_FOR_PIECES(i, col, left)
            {
                affine(v[i], r, p.post_weight, p.post_bias, col, left);
                float g[PIECE];
                if (p.d.gate >= MMM_GATE_COL)
                    mmm_load_piece(static_cast<const T *>(p.gate) + (p.d.gate == MMM_GATE_FULL ? row * p.ldgate : 0) + col, left, g);
#pragma unroll
                for (int q = 0; q < PIECE; ++q) {
                    h[i][q] = p.d.alpha * h[i][q] + (p.d.gate >= MMM_GATE_COL ? g[q] : row_gate) * v[i][q];
                    if (q >= left) h[i][q] = 0.f;
                }
                if (p.h_out != nullptr) mmm_store_piece(static_cast<TH *>(p.h_out) + row * p.ldh_out + col, left, h[i]);
            }
        }
        if (p.d.pre != MMM_NORM_NONE) {
            const float r = standard(h, p.d.pre, 1);
            MMM_FOR_PIECES(i, col, left)
            {
                affine(h[i], r, p.pre_weight, p.pre_bias, col, left);
                mmm_store_piece(static_cast<T *>(p.n) + row * p.ldn + col, left, h[i]);
            }
        }
    }
}

// sums over rows, in this order in the workspace
enum { SUM_PRE_WEIGHT, SUM_PRE_BIAS, SUM_POST_WEIGHT, SUM_POST_BIAS, SUM_GATE, SUMS };

struct NormGradParams {
    mmm_block_norm_desc d;
    mmm_block_norm_grads g;
    float inv_n;
    float *partials;        // [workgroup][sum asked for][N]
    int32_t place[SUMS];    // of a sum among those asked for; -1: not asked for
    int32_t sums;
};

template <typename T, typename TH, typename TY, int V> __global__ __launch_bounds__(1024) void mmm_block_norm_grad_kernel(const NormGradParams p)
{
    __shared__ float rooms[2][4][48];   // (rows in turn, as above)
    const mmm_block_norm_grads &g = p.g;
    const int N = (int)p.d.N, waves = (int)blockDim.x >> 6;
    const bool pre = p.d.pre != MMM_NORM_NONE, block = g.y != nullptr, post = p.d.post != MMM_NORM_NONE;
    const bool pre_mean = p.d.pre == MMM_NORM_LAYER, post_mean = p.d.post == MMM_NORM_LAYER;
    float sums[SUMS][V][PIECE];
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int q = 0; q < PIECE; ++q) sums[s][i][q] = 0.f;

    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.d.M; row += gridDim.x, turn ^= 1) {
        float x[V][PIECE], dn[V][PIECE], d[V][PIECE], y[V][PIECE];
        MMM_FOR_PIECES(i, col, left)
        {
            if (pre) {
                mmm_load_piece(static_cast<const TH *>(g.h_out) + row * g.ldh_out + col, left, x[i]);
                mmm_load_piece(static_cast<const T *>(g.d_n) + row * g.ldd_n + col, left, dn[i]);
            }
            if (g.d_h_out != nullptr)
                mmm_load_piece(static_cast<const TH *>(g.d_h_out) + row * g.ldd_h_out + col, left, d[i]);
            else
#pragma unroll
                for (int q = 0; q < PIECE; ++q) d[i][q] = 0.f;
            if (block) mmm_load_piece(static_cast<const TY *>(g.y) + row * g.ldy + col, left, y[i]);
        }
        // both rows standardised together: one sum for means, one for variances
        float s2[2] = {0.f, 0.f};
        if (pre_mean || post_mean) {
            MMM_FOR_PIECES(i, col, left)
            {
#pragma unroll
                for (int q = 0; q < PIECE; ++q) {
                    if (pre_mean) s2[0] += x[i][q];
                    if (post_mean) s2[1] += y[i][q];
                }
            }
            add_over_row(s2, rooms[turn][0], waves);
            const float mx = pre_mean ? s2[0] * p.inv_n : 0.f, my = post_mean ? s2[1] * p.inv_n : 0.f;
            MMM_FOR_PIECES(i, col, left)
            {
#pragma unroll
                for (int q = 0; q < PIECE; ++q) {
                    if (pre_mean) x[i][q] = q < left ? x[i][q] - mx : 0.f;
                    if (post_mean) y[i][q] = q < left ? y[i][q] - my : 0.f;
                }
            }
            s2[0] = s2[1] = 0.f;
        }
        MMM_FOR_PIECES(i, col, left)
        {
#pragma unroll
            for (int q = 0; q < PIECE; ++q) {
                if (pre) s2[0] += x[i][q] * x[i][q];
                if (post) s2[1] += y[i][q] * y[i][q];
            }
        }
        if (pre || post) add_over_row(s2, rooms[turn][1], waves);
        const float rx = 1.f / sqrtf(s2[0] * p.inv_n + p.d.eps), ry = 1.f / sqrtf(s2[1] * p.inv_n + p.d.eps);
        // through the norm in front of the next block: d becomes the gradient of h'
        if (pre) {
            float c[2] = {0.f, 0.f};
            MMM_FOR_PIECES(i, col, left)
            {
                float w[PIECE];
                if (g.pre_weight != nullptr) mmm_load_piece(static_cast<const T *>(g.pre_weight) + col, left, w);
#pragma unroll
                for (int q = 0; q < PIECE; ++q) {
                    x[i][q] *= rx;
                    if (p.place[SUM_PRE_WEIGHT] >= 0) sums[SUM_PRE_WEIGHT][i][q] += dn[i][q] * x[i][q];
                    if (p.place[SUM_PRE_BIAS] >= 0) sums[SUM_PRE_BIAS][i][q] += dn[i][q];
                    if (g.pre_weight != nullptr) dn[i][q] *= w[q];
                    c[0] += dn[i][q] * x[i][q];
                    c[1] += dn[i][q];
                }
            }
            add_over_row(c, rooms[turn][2], waves);
            const float along = c[0] * p.inv_n, mean = pre_mean ? c[1] * p.inv_n : 0.f;
            MMM_FOR_PIECES(i, col, left)
            {
#pragma unroll
                for (int q = 0; q < PIECE; ++q) d[i][q] += rx * (dn[i][q] - x[i][q] * along - mean);
            }
        }
        if (g.d_h != nullptr) {
            const float alpha = block ? p.d.alpha : 1.f;
            MMM_FOR_PIECES(i, col, left)
            {
                float out[PIECE];
#pragma unroll
                for (int q = 0; q < PIECE; ++q) out[q] = alpha * d[i][q];
                mmm_store_piece(static_cast<TH *>(g.d_h) + row * g.ldd_h + col, left, out);
            }
        }
        if (!block) continue;   // (uniform: no sum is under way)
        // through gate and norm behind the block: d becomes the gradient of y
        const float row_gate = p.d.gate == MMM_GATE_ROW ? (float)static_cast<const T *>(g.gate_values)[row] : 1.f;
        float c[3] = {0.f, 0.f, 0.f};
        MMM_FOR_PIECES(i, col, left)
        {
            float gate[PIECE], w[PIECE], b[PIECE], dgate[PIECE];
            if (p.d.gate >= MMM_GATE_COL)
                mmm_load_piece(static_cast<const T *>(g.gate_values) + (p.d.gate == MMM_GATE_FULL ? row * g.ldgate : 0) + col, left, gate);
            if (g.post_weight != nullptr) mmm_load_piece(static_cast<const T *>(g.post_weight) + col, left, w);
            if (g.post_bias != nullptr) mmm_load_piece(static_cast<const T *>(g.post_bias) + col, left, b);
#pragma unroll
            for (int q = 0; q < PIECE; ++q) {
                if (q >= left) d[i][q] = 0.f;   // (past the row; the mean has been taken off there, too)
                if (post) y[i][q] *= ry;
                float v = y[i][q];
                if (g.post_weight != nullptr) v *= w[q];
                if (g.post_bias != nullptr) v += b[q];
                dgate[q] = d[i][q] * v;
                c[2] += dgate[q];
                if (p.place[SUM_GATE] >= 0) sums[SUM_GATE][i][q] += dgate[q];
                d[i][q] *= p.d.gate >= MMM_GATE_COL ? gate[q] : row_gate;
                if (p.place[SUM_POST_WEIGHT] >= 0) sums[SUM_POST_WEIGHT][i][q] += d[i][q] * y[i][q];
                if (p.place[SUM_POST_BIAS] >= 0) sums[SUM_POST_BIAS][i][q] += d[i][q];
                if (g.post_weight != nullptr) d[i][q] *= w[q];
                c[0] += d[i][q] * y[i][q];
                c[1] += d[i][q];
            }
            if (p.d.gate == MMM_GATE_FULL && g.d_gate != nullptr)
                mmm_store_piece(static_cast<T *>(g.d_gate) + row * g.ldd_gate + col, left, dgate);
        }
        const bool row_sum = p.d.gate == MMM_GATE_ROW && g.d_gate != nullptr;
        if (post || row_sum) add_over_row(c, rooms[turn][3], waves);
        if (row_sum && threadIdx.x == 0) static_cast<float *>(g.d_gate)[row] = c[2];
        if (g.d_y != nullptr) {
            const float along = c[0] * p.inv_n, mean = post_mean ? c[1] * p.inv_n : 0.f;
            MMM_FOR_PIECES(i, col, left)
            {
                if (post)
#pragma unroll
                    for (int q = 0; q < PIECE; ++q) d[i][q] = ry * (d[i][q] - y[i][q] * along - mean);
                mmm_store_piece(static_cast<TY *>(g.d_y) + row * g.ldd_y + col, left, d[i]);
            }
        }
    }
    if (p.sums == 0) return;
#pragma unroll
    for (int s = 0; s < SUMS; ++s) {
        if (p.place[s] < 0) continue;
        MMM_FOR_PIECES(i, col, left) mmm_store_piece(p.partials + ((int64_t)blockIdx.x * p.sums + p.place[s]) * N + col, left, sums[s][i]);
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
#pragma unroll
                for (int q = 0; q < PIECE; ++q) d[q] *= mmm_slope(z[q], p.activation);
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

// Partial sums added in order: out[s][j] = sum over g of partials[g][s][j].  Sixteen waves take every sixteenth g each.
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
        const int64_t col = col0 + lane;
        float sum = 0.f;
        if (col < p.N)
            for (int64_t g = wave; g < p.groups; g += REDUCE_WAVES) sum += p.partials[(g * p.sums + s) * p.N + col];
        room[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && col < p.N) {
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

// Threads and pieces per lane for a row: one piece as long as a workgroup has room.
struct RowShape { uint32_t threads; int pieces; };
RowShape row_shape(int64_t N, uint32_t most)
{
    const uint32_t lanes = (uint32_t)((N + PIECE - 1) / PIECE);
    const int pieces = lanes <= most ? 1 : lanes <= 2 * most ? 2 : 4;
    const uint32_t threads = ((lanes + (uint32_t)pieces - 1) / (uint32_t)pieces + 63) / 64 * 64;
    return {threads, pieces};
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

int64_t norm_grad_groups(int64_t M) { return std::min<int64_t>(M, 512); }
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
    const RowShape shape = row_shape(d.N, 1024);
    if (d.M < 1 || d.N < 1 || d.N > MMM_NORM_MAX_WIDTH) return hipErrorInvalidValue;
    const NormParams p{d, 1.f / (float)d.N, h, y, gate, post_weight, post_bias, pre_weight, pre_bias, ldh, ldy, ldgate, h_out, n, ldh_out, ldn};
    (void)hipGetLastError();
    with_types(d, [&](auto t, auto th, auto ty) {
        typedef decltype(t) T;
        typedef decltype(th) TH;
        typedef decltype(ty) TY;
        void (*fn)(const NormParams) = shape.pieces == 1   ? mmm_block_norm_kernel<T, TH, TY, 1>
                                       : shape.pieces == 2 ? mmm_block_norm_kernel<T, TH, TY, 2>
                                                           : mmm_block_norm_kernel<T, TH, TY, 4>;
        hipLaunchKernelGGL(fn, dim3((uint32_t)std::min(d.M, MAX_GROUPS)), dim3(shape.threads), 0, s, p);
        return 0;
    });
    return hipGetLastError();
}

size_t mmm_block_norm_grad_bytes(int64_t M, int64_t N) { return (size_t)norm_grad_groups(M) * (size_t)N * SUMS * sizeof(float); }

hipError_t mmm_launch_block_norm_grad(const mmm_block_norm_desc &d, const mmm_block_norm_grads &g, void *workspace, hipStream_t s)
{
    const RowShape shape = row_shape(d.N, 1024);
    if (d.M < 1 || d.N < 1 || d.N > MMM_NORM_MAX_WIDTH) return hipErrorInvalidValue;
    NormGradParams p{d, g, 1.f / (float)d.N, static_cast<float *>(workspace), {}, 0};
    float *const out[SUMS] = {g.d_pre_weight, g.d_pre_bias, g.d_post_weight, g.d_post_bias, d.gate == MMM_GATE_COL ? static_cast<float *>(g.d_gate) : nullptr};
    const int64_t groups = norm_grad_groups(d.M);
    ReduceParams r{p.partials, groups, d.N, 0, {}};
    for (int q = 0; q < SUMS; ++q) {
        p.place[q] = out[q] != nullptr ? r.sums : -1;
        if (out[q] != nullptr) r.out[r.sums++] = out[q];
    }
    p.sums = r.sums;
    (void)hipGetLastError();
    with_types(d, [&](auto t, auto th, auto ty) {
        typedef decltype(t) T;
        typedef decltype(th) TH;
        typedef decltype(ty) TY;
        void (*fn)(const NormGradParams) = shape.pieces == 1   ? mmm_block_norm_grad_kernel<T, TH, TY, 1>
                                           : shape.pieces == 2 ? mmm_block_norm_grad_kernel<T, TH, TY, 2>
                                                               : mmm_block_norm_grad_kernel<T, TH, TY, 4>;
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
