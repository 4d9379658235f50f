// The multiplication on matrix instructions with bias, activation and residual on the way to C: instances of the kernel of
// mmm_matmul_kernel.h, and the sum of the partial products of a split K, behind which the epilogue comes.
//
// The epilogue costs what it reads and writes: applied to the accumulators it saves a pass over C in float for each of bias,
// activation, residual and conversion.
#include <algorithm>

#include "mmm_matmul_kernel.h"

namespace {

// As mmm_splitk_reduce_kernel, in the same order; a lane's neighbours exist all or none (N is a multiple of 8).
template <typename E, typename T>
__global__ __launch_bounds__(256) void mmm_splitk_epilogue_kernel(const E *P, void *C, int64_t ldc, uint32_t M, uint32_t NV, int32_t splits,
                                                                  const mmm_epilogue_args epilogue)
{
    constexpr int VEC = 16 / (int)sizeof(E);
    typedef E vec __attribute__((ext_vector_type(VEC)));
    const vec *parts = reinterpret_cast<const vec *>(P);
    const uint32_t col = blockIdx.x * 256u + threadIdx.x;
    if (col >= NV) return;
    const int64_t total = (int64_t)M * NV;
    mmm_column_values<T, E, VEC> columns;
    columns.load(epilogue, (int64_t)col * VEC);
    for (uint32_t row = blockIdx.y; row < M; row += gridDim.y) {
        const int64_t e = (int64_t)row * NV + col;
        E more[VEC];
        columns.residual(epilogue, row, (int64_t)col * VEC, more);
        vec sum = parts[e];
        for (int32_t sp = 1; sp < splits; sp += 8) {
            vec v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = sp + i < splits ? parts[(int64_t)(sp + i) * total + e] : vec(0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (sp + i < splits) sum += v[i];
        }
        E z[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) z[q] = sum[q];
        columns.activate(epilogue, z, row, (int64_t)col * VEC);
        columns.finish(epilogue, z, more, C, ldc, row, (int64_t)col * VEC);
    }
}

}   // namespace

hipError_t mmm_launch_matmul_epilogue(const mmm_maps *m, const mmm_plan &pl, int32_t dtype, void *C, int64_t ldc, const mmm_epilogue_args &epilogue,
                                      void *partials, size_t partial_bytes, hipStream_t s)
{
    if (pl.split_k <= 1) return launch_tiles<true>(m, pl, dtype, C, ldc, 0, epilogue, nullptr, 0, s);
    if (hipError_t e = mmm_launch_tiles(m, pl, dtype, nullptr, 0, 0, partials, partial_bytes, s); e != hipSuccess) return e;
    const uint32_t NV = (uint32_t)(m->N / (dtype == MMM_F64 ? 2 : 4));
    const dim3 grid((NV + 255) / 256, (uint32_t)std::min<int64_t>(m->M, 65535));
    if (dtype == MMM_F64)
        hipLaunchKernelGGL((mmm_splitk_epilogue_kernel<double, double>), grid, dim3(256), 0, s, static_cast<const double *>(partials), C, ldc, (uint32_t)m->M, NV,
                           pl.split_k, epilogue);
    else
        hipLaunchKernelGGL((dtype == MMM_BF16  ? mmm_splitk_epilogue_kernel<float, __bf16>
                            : dtype == MMM_F16 ? mmm_splitk_epilogue_kernel<float, _Float16>
                                               : mmm_splitk_epilogue_kernel<float, float>),
                           grid, dim3(256), 0, s, static_cast<const float *>(partials), C, ldc, (uint32_t)m->M, NV, pl.split_k, epilogue);
    return hipGetLastError();
}
