// The norm of all gradients and the AdamW step, over a table of tensors. A warp takes one block of FTC_STATE_BLOCK elements of one
// tensor at a time, 8 elements a lane; the table gives it the block's tensor.
#include "ftc_train.cuh"

namespace ftc {

constexpr uint32_t kWarps = 8;
constexpr float kTiny = 1.1754943508222875e-38f;                 // 2^-126, the smallest scale
constexpr float kInv127 = 1.0f / 16129.0f, kInv255 = 1.0f / 65025.0f;

__device__ __forceinline__ float load_f32(const void* p, uint32_t dtype, uint64_t i) {
    if (dtype == FTC_F32) return static_cast<const float*>(p)[i];
    if (dtype == FTC_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_f32(void* p, uint32_t dtype, uint64_t i, float v) {
    if (dtype == FTC_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == FTC_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(v);
    else static_cast<__half*>(p)[i] = from_f32<__half>(v);
}

// 1 / processes included in the message of element i, 0 where it was not delivered.
__device__ __forceinline__ float share(const TableEntry& t, uint64_t i) {
    if (!t.status) return 1.f;
    const uint2 s = *reinterpret_cast<const uint2*>(t.status + i / t.k * FTC_STATUS_WORDS);
    return (s.x & 0xFFu) == FTC_ST_OK && s.y ? 1.f / (float)s.y : 0.f;
}

// The whole number c with (c - 1/2)^2 <= x < (c + 1/2)^2, at most `most`. The squares are exact in float32, so the result does not
// depend on how the root is rounded.
__device__ __forceinline__ float nearest_root(float x, float most) {
    float c = floorf(sqrtf(x) + 0.5f);
    if (c * c - c + 0.25f > x) c -= 1.f;
    if (c * c + c + 0.25f <= x) c += 1.f;
    return fminf(fmaxf(c, 0.f), most);
}

// Largest of the warp's non-negative values, as bit patterns: infinities above all numbers, NaN above them.
__device__ __forceinline__ float warp_max_bits(float v) {
    return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v) & 0x7FFFFFFFu));
}

template <int BITS>
__global__ void __launch_bounds__(kWarps * 32) adamw_kernel(AdamArgs a) {
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t b = blockIdx.x * (uint64_t)kWarps + (threadIdx.x >> 5);
    if (b >= a.n_blocks) return;
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!isfinite(scale)) return;
    const TableEntry t = table_entries(a.table)[table_map(a.table, a.n_params)[b]];
    const float lr = a.lr * t.lr_scale, keep = 1.f - lr * t.weight_decay, rate = lr * a.fix1;
    const uint64_t e0 = (b - t.first_block) * FTC_STATE_BLOCK;
    float m[8], v[8];
    bool there[8];
    bool some = false;
    const float ms = BITS == 8 ? a.m_scale[b] * kInv127 : 0.f, vs = BITS == 8 ? a.v_scale[b] * kInv255 : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint64_t i = e0 + j * 32 + lane, q = b * FTC_STATE_BLOCK + j * 32 + lane;
        if (BITS == 32) { m[j] = static_cast<const float*>(a.m)[q]; v[j] = static_cast<const float*>(a.v)[q]; }
        else {
            const float c = (float)static_cast<const int8_t*>(a.m)[q], d = (float)static_cast<const uint8_t*>(a.v)[q];
            m[j] = c * fabsf(c) * ms;
            const float r = d * d * vs;
            v[j] = r * r;
        }
        there[j] = false;
        if (i < t.n) {
            const float w = share(t, i);
            if (w > 0.f) {
                there[j] = some = true;
                const float g = load_f32(t.grad, t.grad_dtype, i) * w * scale;
                m[j] = m[j] * a.beta1 + g * a.rest1;
                v[j] = v[j] * a.beta2 + g * g * a.rest2;
                float p = t.master ? t.master[i] : load_f32(t.param, t.param_dtype, i);
                p = p * keep - m[j] / (sqrtf(v[j]) * a.fix2 + a.eps) * rate;
                if (t.master) t.master[i] = p;
                store_f32(t.param, t.param_dtype, i, p);
            }
        }
    }
    if (BITS == 32) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (there[j]) {
                const uint64_t q = b * FTC_STATE_BLOCK + j * 32 + lane;
                static_cast<float*>(a.m)[q] = m[j];
                static_cast<float*>(a.v)[q] = v[j];
            }
        return;
    }
    if (!__any_sync(0xFFFFFFFFu, some)) return;
    float mm = 0.f, rm = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = sqrtf(v[j]);
        mm = __uint_as_float(max(__float_as_uint(mm), __float_as_uint(m[j]) & 0x7FFFFFFFu));
        rm = __uint_as_float(max(__float_as_uint(rm), __float_as_uint(v[j]) & 0x7FFFFFFFu));
    }
    mm = warp_max_bits(mm); rm = warp_max_bits(rm);
    mm = mm < kTiny ? kTiny : mm; rm = rm < kTiny ? kTiny : rm;             // NaN stays
    const float mi = 1.f / mm, ri = 1.f / rm;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint64_t q = b * FTC_STATE_BLOCK + j * 32 + lane;
        const float c = nearest_root(fabsf(m[j]) * mi * 16129.f, 127.f);
        float d = nearest_root(v[j] * ri * 65025.f, 255.f);
        if (v[j] > 0.f) d = fmaxf(d, 1.f);
        static_cast<int8_t*>(a.m)[q] = (int8_t)(int)(m[j] < 0.f ? -c : c);
        static_cast<uint8_t*>(a.v)[q] = (uint8_t)(int)d;
    }
    if (lane == 0) { a.m_scale[b] = mm; a.v_scale[b] = rm; }
}

cudaError_t launch_adamw(const AdamArgs& a, int, cudaStream_t st) {
    const uint32_t grid = (uint32_t)((a.n_blocks + kWarps - 1) / kWarps);
    if (a.bits == 32) adamw_kernel<32><<<grid, kWarps * 32, 0, st>>>(a);
    else adamw_kernel<8><<<grid, kWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}

__global__ void __launch_bounds__(256) adamw_states_kernel(uint64_t n, const int8_t* m, const uint8_t* v, const float* ms, const float* vs, float* mo, float* vo) {
    const uint64_t i = blockIdx.x * 256ull + threadIdx.x;                       // one block of the states for each thread block
    const float c = (float)m[i], d = (float)v[i], r = d * d * (vs[blockIdx.x] * kInv255);
    mo[i] = c * fabsf(c) * (ms[blockIdx.x] * kInv127);
    vo[i] = r * r;
}

cudaError_t launch_adamw_states(uint64_t blocks, const void* m, const void* v, const float* ms, const float* vs, float* mo, float* vo, int, cudaStream_t st) {
    for (uint64_t at = 0; at < blocks; at += 1u << 30) {
        const uint64_t n = blocks - at < (1u << 30) ? blocks - at : 1u << 30, e = at * FTC_STATE_BLOCK;
        adamw_states_kernel<<<(uint32_t)n, 256, 0, st>>>(n, static_cast<const int8_t*>(m) + e, static_cast<const uint8_t*>(v) + e, ms + at, vs + at, mo + e, vo + e);
    }
    return cudaGetLastError();
}

// ---- the norm: warp w adds up the squares of the blocks [w*span, (w+1)*span) and leaves one sum for each tensor it meets; warp w and
// tensor t share slot w + t (going on by one block either grows, so no two pairs with blocks in common share a slot)

__global__ void __launch_bounds__(kWarps * 32) grad_squares_kernel(const void* table, uint32_t n_params, uint64_t n_blocks, uint64_t span, double* slots) {
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t w = blockIdx.x * (uint64_t)kWarps + (threadIdx.x >> 5), b0 = w * span, b1 = b0 + span < n_blocks ? b0 + span : n_blocks;
    const uint32_t* map = table_map(table, n_params);
    double s = 0;
    for (uint64_t b = b0; b < b1; ++b) {
        const uint32_t ti = map[b];
        const TableEntry t = table_entries(table)[ti];
        for (int j = 0; j < 8; ++j) {
            const uint64_t i = (b - t.first_block) * FTC_STATE_BLOCK + j * 32 + lane;
            if (i < t.n) {
                const float w8 = share(t, i);
                if (w8 > 0.f) { const double g = load_f32(t.grad, t.grad_dtype, i) * w8; s += g * g; }
            }
        }
        if (b + 1 == b1 || map[b + 1] != ti) {
            s = warp_sum(s);
            if (lane == 0) slots[w + ti] = s;
            s = 0;
        }
    }
}

// One block: a warp for each tensor's sum, then the sum over tensors.
__global__ void __launch_bounds__(1024) grad_norm_kernel(const void* table, uint32_t n_params, uint64_t span, float max_norm, const double* slots, double* sums,
                                                         float* norm, float* norms) {
    __shared__ double part[32];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t ti = warp; ti < n_params; ti += 32) {
        const TableEntry& t = table_entries(table)[ti];
        double s = 0;
        if (t.n) {
            const uint64_t last = t.first_block + (t.n - 1) / FTC_STATE_BLOCK;
            for (uint64_t w = t.first_block / span + lane; w <= last / span; w += 32) s += slots[w + ti];
        }
        s = warp_sum(s);
        if (lane == 0) { sums[ti] = s; if (norms) norms[ti] = (float)sqrt(s); }
    }
    __syncthreads();
    double s = 0;
    for (uint32_t ti = threadIdx.x; ti < n_params; ti += 1024) s += sums[ti];
    s = warp_sum(s);
    if (lane == 0) part[warp] = s;
    __syncthreads();
    if (warp == 0) {
        s = warp_sum(part[lane]);
        if (lane == 0) {
            const float r = (float)sqrt(s);
            norm[0] = r;
            norm[1] = !isfinite(r) ? __uint_as_float(0x7FC00000u) : r > max_norm ? max_norm / r : 1.f;
        }
    }
}

// Warps that share the blocks: at most those the GPU holds.
uint32_t grad_norm_warps(uint64_t n_blocks, int sm_count) {
    const uint64_t cap = (uint64_t)sm_count * 48;
    return (uint32_t)(n_blocks < cap ? n_blocks : cap);
}

cudaError_t launch_grad_norm(const void* table, uint32_t n_params, uint64_t n_blocks, float max_norm, float* norm, float* norms, double* ws, int sm_count,
                             cudaStream_t st) {
    const uint32_t warps = grad_norm_warps(n_blocks, sm_count);
    const uint64_t span = warps ? (n_blocks + warps - 1) / warps : 1;
    double* sums = ws + warps + n_params;
    if (warps) {
        grad_squares_kernel<<<(warps + kWarps - 1) / kWarps, kWarps * 32, 0, st>>>(table, n_params, n_blocks, span, ws);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    grad_norm_kernel<<<1, 1024, 0, st>>>(table, n_params, span, max_norm, ws, sums, norm, norms);
    return cudaGetLastError();
}

}  // namespace ftc
