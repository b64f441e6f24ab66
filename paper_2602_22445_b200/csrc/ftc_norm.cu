// Layer norm forward and backward, with the weight gradients of each process of a data-parallel job.
//
// A thread block walks rows; the sums over a row are taken by the whole block. The weight gradients are sums over rows: block
// b walks the rows [b*R, (b+1)*R) in order and keeps one partial sum per column, which it leaves in the workspace whenever
// the row's process changes and at its end. Block b and process p share slot b + p: going on by one row either the block or
// the process grows, so no two (block, process) pairs that have rows in common meet in one slot, and blocks + P slots are enough
// however the rows are divided. A second kernel adds the slots of each process in ascending order and lays the sums out as messages.
#include "ftc_train.cuh"

namespace ftc {

constexpr uint32_t kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* scratch) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
    for (uint32_t i = 0; i < kThreads / 32; ++i) s += scratch[i];
    return s;
}

template <typename T, typename W>
__global__ void __launch_bounds__(kThreads) norm_forward_kernel(NormArgs a) {
    __shared__ float scratch[kThreads / 32];
    const W* gamma = static_cast<const W*>(a.gamma);
    const W* beta = static_cast<const W*>(a.beta);
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        T* y = static_cast<T*>(a.y) + r * a.y_stride;
        float s = 0.f;
        for (uint32_t h = threadIdx.x; h < a.H; h += kThreads) s += to_f32(x[h]);
        const float mean = block_sum(s, scratch) / a.H;
        s = 0.f;
        for (uint32_t h = threadIdx.x; h < a.H; h += kThreads) { const float d = to_f32(x[h]) - mean; s = fmaf(d, d, s); }
        const float rstd = 1.f / sqrtf(block_sum(s, scratch) / a.H + a.eps);
        for (uint32_t h = threadIdx.x; h < a.H; h += kThreads)
            y[h] = from_f32<T>((to_f32(x[h]) - mean) * rstd * (gamma ? to_f32(gamma[h]) : 1.f) + (beta ? to_f32(beta[h]) : 0.f));
        if (threadIdx.x == 0) {
            if (a.mean_out) a.mean_out[r] = mean;
            if (a.rstd_out) a.rstd_out[r] = rstd;
        }
    }
}

// First row of process p, at most `rows`.
__device__ __forceinline__ uint64_t first_row(const NormArgs& a, uint64_t p) {
    if (!a.splits) return p * a.rows / a.P;
    const uint64_t s = a.splits[p];
    return s < a.rows ? s : a.rows;
}

// The process that holds row r: the first one that ends behind it (P if none does).
__device__ __forceinline__ uint32_t holder(const NormArgs& a, uint64_t r) {
    uint32_t lo = 0, hi = a.P;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (first_row(a, (uint64_t)mid + 1) > r) hi = mid; else lo = mid + 1;
    }
    return lo;
}

template <typename T, typename W>
__global__ void __launch_bounds__(kThreads) norm_backward_kernel(NormArgs a) {
    __shared__ float scratch[kThreads / 32];
    const W* gamma = static_cast<const W*>(a.gamma);
    const uint64_t r0 = blockIdx.x * a.rows_per_block, r1 = r0 + a.rows_per_block < a.rows ? r0 + a.rows_per_block : a.rows;
    uint32_t p = a.slots ? holder(a, r0) : 0;
    uint64_t end = a.slots && p < a.P ? first_row(a, (uint64_t)p + 1) : 0;
    bool fresh = true;
    for (uint64_t r = r0; r < r1; ++r) {
        while (p < a.P && a.slots && r >= end) { ++p; fresh = true; end = p < a.P ? first_row(a, (uint64_t)p + 1) : 0; }
        const bool counts = a.slots && p < a.P && r >= first_row(a, p);
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + r * a.dy_stride;
        T* dx = static_cast<T*>(a.dx) + r * a.dx_stride;
        float* dg = a.slots + ((uint64_t)blockIdx.x + p) * 2 * a.H;
        float* db = dg + a.H;
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s1 = 0.f, s2 = 0.f;
        for (uint32_t h = threadIdx.x; h < a.H; h += kThreads) {
            const float g = to_f32(dy[h]), xh = (to_f32(x[h]) - mean) * rstd, u = g * (gamma ? to_f32(gamma[h]) : 1.f);
            s1 += u; s2 = fmaf(u, xh, s2);
            if (counts) { dg[h] = fresh ? g * xh : dg[h] + g * xh; db[h] = fresh ? g : db[h] + g; }
        }
        if (counts) fresh = false;
        if (!a.dx) continue;
        const float c1 = block_sum(s1, scratch) / a.H, c2 = block_sum(s2, scratch) / a.H;
        for (uint32_t h = threadIdx.x; h < a.H; h += kThreads) {
            const float xh = (to_f32(x[h]) - mean) * rstd, u = to_f32(dy[h]) * (gamma ? to_f32(gamma[h]) : 1.f);
            dx[h] = from_f32<T>(rstd * (u - c1 - xh * c2));
        }
    }
}

// dgamma[s][p][e], dbeta[s][p][e] from the slots: a thread for each element.
__global__ void __launch_bounds__(kThreads) norm_messages_kernel(NormArgs a) {
    const uint64_t S = (a.H + a.k - 1) / a.k, n = S * a.P * a.k;
    for (uint64_t i = blockIdx.x * (uint64_t)kThreads + threadIdx.x; i < n; i += (uint64_t)gridDim.x * kThreads) {
        const uint64_t e = i % a.k, p = i / a.k % a.P, h = i / a.k / a.P * a.k + e;
        float g = 0.f, b = 0.f;
        const uint64_t lo = first_row(a, p), hi = first_row(a, p + 1);
        if (h < a.H && lo < hi)
            for (uint64_t blk = lo / a.rows_per_block; blk <= (hi - 1) / a.rows_per_block; ++blk) {
                g += a.slots[(blk + p) * 2 * a.H + h];
                b += a.slots[(blk + p) * 2 * a.H + a.H + h];
            }
        if (a.dgamma) a.dgamma[i] = g;
        if (a.dbeta) a.dbeta[i] = b;
    }
}

template <typename F> static cudaError_t by_type(uint32_t dtype, uint32_t wdtype, F f) {
    if (dtype == FTC_F32) f(float(), float());
    else if (dtype == FTC_BF16) { if (wdtype == FTC_F32) f(__nv_bfloat16(), float()); else f(__nv_bfloat16(), __nv_bfloat16()); }
    else { if (wdtype == FTC_F32) f(__half(), float()); else f(__half(), __half()); }
    return cudaGetLastError();
}

cudaError_t launch_norm_forward(const NormArgs& a, int sm_count, cudaStream_t st) {
    const uint64_t cap = (uint64_t)sm_count * 8;
    const uint32_t grid = (uint32_t)(a.rows < cap ? a.rows : cap);
    return by_type(a.dtype, a.wdtype, [&](auto t, auto w) { norm_forward_kernel<decltype(t), decltype(w)><<<grid, kThreads, 0, st>>>(a); });
}

// As many blocks as the GPU holds, fewer where their partial sums would take up more than 2 GiB.
uint32_t norm_backward_blocks(uint32_t H, uint64_t rows, int sm_count) {
    uint64_t b = (uint64_t)sm_count * 4;
    const uint64_t room = (1ull << 28) / H;
    if (b > room) b = room ? room : 1;
    if (b > rows) b = rows;
    if (b == 0) return 0;
    const uint64_t each = (rows + b - 1) / b;
    return (uint32_t)((rows + each - 1) / each);
}

cudaError_t launch_norm_backward(NormArgs a, cudaStream_t st) {
    cudaError_t e;
    if (a.blocks) {
        e = by_type(a.dtype, a.wdtype, [&](auto t, auto w) { norm_backward_kernel<decltype(t), decltype(w)><<<a.blocks, kThreads, 0, st>>>(a); });
        if (e != cudaSuccess) return e;
    }
    if (!a.slots) return cudaSuccess;
    const uint64_t n = (uint64_t)((a.H + a.k - 1) / a.k) * a.P * a.k, want = (n + kThreads - 1) / kThreads;
    norm_messages_kernel<<<(uint32_t)(want < 65536 ? want : 65536), kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace ftc
