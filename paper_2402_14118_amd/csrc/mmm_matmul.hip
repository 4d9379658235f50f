// The multiplication on matrix instructions: instances of the kernel of mmm_matmul_kernel.h for the plain product, and the launch.
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "mmm_matmul_kernel.h"

namespace {

// Sum of the split-K partials in a fixed order (split 0, 1, ...), so the result
// does not depend on the order in which workgroups finish.  Bound by latency: a thread takes VEC neighbours of a row, and
// the loads of eight splits are in flight together.
template <typename E, int VEC>
__global__ __launch_bounds__(256) void mmm_splitk_reduce_kernel(const E *P, E *C, int64_t ldc, uint32_t M, uint32_t NV,
                                                                int32_t splits, int32_t accumulate)
{
    typedef E vec __attribute__((ext_vector_type(VEC)));
    typedef vec vec_u __attribute__((aligned(sizeof(E) * VEC)));
    const vec_u *parts = reinterpret_cast<const vec_u *>(P);
    const uint32_t col = blockIdx.x * 256u + threadIdx.x;
    if (col >= NV) return;
    const int64_t total = (int64_t)M * NV;
    for (uint32_t row = blockIdx.y; row < M; row += gridDim.y) {
        const int64_t e = (int64_t)row * NV + col;
        vec sum = parts[e];
        for (int32_t sp = 1; sp < splits; sp += 8) {
            vec v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = sp + i < splits ? parts[(int64_t)(sp + i) * total + e] : vec(0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (sp + i < splits) sum += v[i];
        }
        vec_u *dst = reinterpret_cast<vec_u *>(C + (int64_t)row * ldc + (int64_t)col * VEC);
        *dst = accumulate ? *dst + sum : sum;
    }
}

template <typename E>
void launch_splitk_reduce(const void *P, void *C, int64_t ldc, int64_t M, int64_t N, int32_t splits, int32_t accumulate, hipStream_t s)
{
    constexpr int VEC = 16 / (int)sizeof(E);   // N is a multiple of 8
    const bool vec = reinterpret_cast<uintptr_t>(C) % 16 == 0 && ldc % VEC == 0 && reinterpret_cast<uintptr_t>(P) % 16 == 0;
    const uint32_t NV = (uint32_t)(vec ? N / VEC : N);
    const dim3 grid((NV + 255) / 256, (uint32_t)std::min<int64_t>(M, 65535));
    if (vec)
        hipLaunchKernelGGL((mmm_splitk_reduce_kernel<E, VEC>), grid, dim3(256), 0, s, static_cast<const E *>(P), static_cast<E *>(C), ldc, (uint32_t)M,
                           NV, splits, accumulate);
    else
        hipLaunchKernelGGL((mmm_splitk_reduce_kernel<E, 1>), grid, dim3(256), 0, s, static_cast<const E *>(P), static_cast<E *>(C), ldc, (uint32_t)M,
                           NV, splits, accumulate);
}


}   // namespace

// Partial sums of the split-K multiplication for callers that cannot bring (or let the library
// carve out of a workspace) a buffer of their own: one array per GPU, held until the process
// ends.  Host code never uses the array's name as an address: the device address is looked up
// once per device and that pointer is what kernels and copies get.
static __device__ __align__(256) unsigned char scratch[MMM_STATIC_SCRATCH_BYTES];

hipError_t mmm_static_scratch(float **ptr)
{
    constexpr int kMaxDevices = 64;
    static std::mutex mu;
    static void *addr[kMaxDevices];   // zero-initialised: not looked up yet
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (addr[dev] == nullptr) {   // the current device's own copy of the array
        void *q = nullptr;
        e = hipGetSymbolAddress(&q, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return e;
        if (q == nullptr) return hipErrorInvalidSymbol;
        addr[dev] = q;
    }
    *ptr = static_cast<float *>(addr[dev]);
    return hipSuccess;
}

int32_t mmm_variant_count() { return VARIANTS; }
const mmm_variant_info &mmm_variant(int32_t i) { return variants<false>()[i].info; }

hipError_t mmm_launch_tiles(const mmm_maps *m, const mmm_plan &pl, int32_t dtype, void *C, int64_t ldc, int32_t accumulate, void *partials,
                            size_t partial_bytes, hipStream_t s)
{
    return launch_tiles<false>(m, pl, dtype, C, ldc, accumulate, {}, partials, partial_bytes, s);
}

hipError_t mmm_launch_matmul(const mmm_maps *m, const mmm_plan &pl, int32_t dtype, void *C, int64_t ldc, int32_t accumulate, void *partials,
                             size_t partial_bytes, hipStream_t s)
{
    const hipError_t e = mmm_launch_tiles(m, pl, dtype, C, ldc, accumulate, partials, partial_bytes, s);
    if (e != hipSuccess || pl.split_k <= 1) return e;
    if (dtype == MMM_F64)
        launch_splitk_reduce<double>(partials, C, ldc, m->M, m->N, pl.split_k, accumulate, s);
    else
        launch_splitk_reduce<float>(partials, C, ldc, m->M, m->N, pl.split_k, accumulate, s);
    return hipGetLastError();
}
