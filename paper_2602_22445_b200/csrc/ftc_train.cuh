// Shared by the training operators: element types, reductions, the table of tensors.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include "../../include/ftc.h"

namespace ftc {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <typename V> __device__ __forceinline__ V warp_sum(V v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Two kernels of one call: the second one may be put on the GPU while the first is at work (all of whose blocks are there at once) and
// waits for its results only where it needs them.
__device__ __forceinline__ void later_kernel_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_earlier_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... A> cudaError_t launch_second(void (*kernel)(A...), dim3 grid, dim3 block, cudaStream_t st, A... args) {
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t how{};
    how.gridDim = grid; how.blockDim = block; how.stream = st; how.attrs = &early; how.numAttrs = 1;
    return cudaLaunchKernelEx(&how, kernel, args...);
}

// ---- the table of tensors: header, entries, one tensor index for each block of FTC_STATE_BLOCK elements ----

constexpr uint64_t kTableMagic = 0x3154424154435446ull;
struct TableHead { uint64_t magic, n_blocks; uint32_t n_params, flags; uint64_t pad; };     // flags bit 0: some tensor has no weights; 1: most blocks are full ones of aligned tensors; 2: neighbours of some tensor's 8 have more than one record
struct TableEntry {
    void* param; float* master; const void* grad; const uint32_t* status;
    uint64_t n, first_block;
    uint32_t k; uint8_t param_dtype, grad_dtype, wide, k_shift;       // k_shift: k = 2^k_shift, or 255
    float lr_scale, weight_decay;
};
static_assert(sizeof(TableHead) == 32 && sizeof(TableEntry) == 64, "table layout");

__host__ __device__ inline const TableEntry* table_entries(const void* t) {
    return reinterpret_cast<const TableEntry*>(static_cast<const char*>(t) + sizeof(TableHead));
}
__host__ __device__ inline const uint32_t* table_map(const void* t, uint32_t n_params) {
    return reinterpret_cast<const uint32_t*>(table_entries(t) + n_params);
}

// launchers (ftc_norm.cu, ftc_optim.cu)
struct NormArgs {
    const void *x, *dy, *gamma, *beta;
    void *y, *dx;
    float *mean_out, *rstd_out;
    const float *mean, *rstd;
    const uint64_t* splits;
    float *dgamma, *dbeta, *slots;
    uint64_t x_stride, y_stride, dy_stride, dx_stride;
    uint32_t rows, H, P, k, dtype, wdtype, groups, rows_per_group, direct;
    float eps;
};
cudaError_t launch_norm_forward(const NormArgs& a, int sm_count, cudaStream_t st);
cudaError_t launch_norm_backward(const NormArgs& a, int sm_count, cudaStream_t st);
// Does each process's group write its messages itself? 2: in vectors of four.
uint32_t norm_backward_direct(const NormArgs& a, int sm_count);
// Groups that share the rows in the backward pass; each leaves its partial sums of the weight gradients in the workspace.
uint32_t norm_backward_groups(uint32_t H, uint64_t rows, int sm_count);

struct AdamArgs {
    const void* table; uint32_t n_params; uint64_t n_blocks;
    void *m, *v; float *m_scale, *v_scale; const float* grad_scale;
    float lr, beta1, beta2, rest1, rest2, eps, fix1, fix2, one;         // one = 1
    uint32_t bits, mostly_wide, dither, phase;                          // phase: step * kDitherStep
};
// Codes rounded up or down by u = (place * kDitherPlace + step * kDitherStep) mod 2^32 / 2^32, with the fractions of sqrt(2) and of the golden
// ratio: over the steps of an element, and over the elements of a step, u takes every part of [0, 1) evenly.
constexpr uint32_t kDitherM = 1, kDitherV = 2, kDitherPlace = 0x6A09E667u, kDitherStep = 0x9E3779B9u;
cudaError_t launch_adamw(const AdamArgs& a, int sm_count, cudaStream_t st);
cudaError_t launch_adamw_states(uint64_t blocks, const void* m, const void* v, const float* ms, const float* vs, float* mo, float* vo, cudaStream_t st);
uint32_t grad_norm_warps(uint64_t n_blocks, int sm_count);
cudaError_t launch_grad_norm(const void* table, uint32_t n_params, uint64_t n_blocks, bool mixed, float max_norm, float* norm, float* norms, double* ws,
                             int sm_count, cudaStream_t st);

}  // namespace ftc
