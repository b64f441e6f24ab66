// Layer norm on rows that fit the registers of a thread block.
//
// A group of G threads (a warp, or a block of up to 1024) holds a row: vector i of thread t is vector i*G + t of the row, so every
// load and store of a warp is one contiguous run. Statistics are taken in two steps from the registers (mean, then squared distances),
// which no common offset of the row can spoil. A group walks many rows with gamma, beta and the column sums in registers, and has the next
// row's loads out while it works on the present one.
#pragma once
#include "ftc_train.cuh"

namespace ftc {

// VB bytes of neighbouring elements, kept as loaded.
template <typename T, int VB> struct Pack {
    static constexpr int N = VB / (int)sizeof(T), WORDS = VB < 4 ? 1 : VB / 4;
    uint32_t r[WORDS];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (VB == 16) { const uint4 v = *reinterpret_cast<const uint4*>(p); r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w; }
        else if constexpr (VB == 4) r[0] = *reinterpret_cast<const uint32_t*>(p);
        else r[0] = *reinterpret_cast<const uint16_t*>(p);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) r[i] = 0u;
    }
    __device__ __forceinline__ float get(int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(r[j]);
        else {
            const uint32_t w = r[j / 2];
            if constexpr (sizeof(T) == 2 && is_bf16()) return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
            else return __half2float(__ushort_as_half((unsigned short)(j & 1 ? w >> 16 : w & 0xFFFFu)));
        }
    }
    static constexpr __host__ __device__ bool is_bf16();
    static __device__ __forceinline__ void store(T* p, const float* v) {
        if constexpr (sizeof(T) == 4) {
            if constexpr (VB == 16) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            else *p = from_f32<T>(v[0]);
        } else if constexpr (VB == 2) *p = from_f32<T>(v[0]);
        else {
            uint32_t w[WORDS];
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if constexpr (is_bf16()) { const __nv_bfloat162 q = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&q); }
                else { const __half2 q = __floats2half2_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&q); }
            }
            if constexpr (VB == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint32_t*>(p) = w[0];
        }
    }
};
template <typename T> struct IsBf16 { static constexpr bool value = false; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr bool value = true; };
template <typename T, int VB> constexpr __host__ __device__ bool Pack<T, VB>::is_bf16() { return IsBf16<T>::value; }

// N weights from column c on; `other` where there are none.
template <typename W, int N> __device__ __forceinline__ void load_weights(float* v, const W* w, uint32_t c, float other) {
    if (!w) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = other;
        return;
    }
    constexpr int BYTES = N * (int)sizeof(W), VB = BYTES >= 16 ? 16 : BYTES == 8 ? 4 : BYTES, M = VB / (int)sizeof(W);
#pragma unroll
    for (int i = 0; i < N / M; ++i) {
        Pack<W, VB> p;
        p.load(w + c + i * M);
#pragma unroll
        for (int j = 0; j < M; ++j) v[i * M + j] = p.get(j);
    }
}

// First row of process p, at most `rows`.
__device__ __forceinline__ uint64_t first_row(const NormArgs& a, uint64_t p) {
    if (!a.splits) return p * a.rows / a.P;
    const uint64_t s = a.splits[p];
    return s < a.rows ? s : a.rows;
}

// The rows of group b, and the process that holds the present one.
struct RowWalk {
    const NormArgs& a;
    uint64_t r0, r1, start, end;
    uint32_t b, p;
    bool any;                                   // the present process has rows here so far
    __device__ __forceinline__ RowWalk(const NormArgs& args, uint32_t group) : a(args), b(group), any(false) {
        r0 = group * a.rows_per_group;
        r1 = r0 + a.rows_per_group < a.rows ? r0 + a.rows_per_group : a.rows;
        if (r0 > r1) r0 = r1;
        uint32_t lo = 0, hi = a.P;              // the first process that ends behind r0 (P if none does)
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (first_row(a, (uint64_t)mid + 1) > r0) hi = mid; else lo = mid + 1;
        }
        p = lo;
        bounds();
    }
    __device__ __forceinline__ void bounds() {
        start = p < a.P ? first_row(a, p) : a.rows;
        end = p < a.P ? first_row(a, (uint64_t)p + 1) : ~0ull;
    }
    __device__ __forceinline__ bool leaves(uint64_t r) const { return r >= end; }
    __device__ __forceinline__ void go_to(uint64_t r) { while (r >= end) { ++p; bounds(); } any = false; }
    __device__ __forceinline__ bool counts(uint64_t r) const { return r >= start && p < a.P; }
    __device__ __forceinline__ uint64_t slot() const { return (uint64_t)b + p; }
};

template <int N> __device__ __forceinline__ void store_slot(const NormArgs& a, uint64_t slot, uint32_t c, const float* dg, const float* db) {
    float* g = a.slots + slot * 2 * a.H + c;
    float* b = g + a.H;
    if constexpr (N % 4 == 0) {                 // N divides H, the workspace begins on 16 bytes
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            *reinterpret_cast<float4*>(g + j) = make_float4(dg[j], dg[j + 1], dg[j + 2], dg[j + 3]);
            *reinterpret_cast<float4*>(b + j) = make_float4(db[j], db[j + 1], db[j + 2], db[j + 3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) { g[j] = dg[j]; b[j] = db[j]; }
    }
}

// Sums over the group. With more than one warp a pair of values goes through shared memory; `turn` alternates between two places, so
// that one barrier a call is enough (a place is written again only behind the barrier of the call in between).
__device__ __forceinline__ float2 group_sum(float2 v, float2 (*scratch)[32], uint32_t& turn) {
#pragma unroll
    for (int o = 16; o; o >>= 1) { v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o); v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o); }
    if (blockDim.x == 32) return v;
    const uint32_t warps = blockDim.x / 32;
    if ((threadIdx.x & 31) == 0) scratch[turn][threadIdx.x >> 5] = v;
    __syncthreads();
    float2 s = scratch[turn][0];
    for (uint32_t i = 1; i < warps; ++i) { s.x += scratch[turn][i].x; s.y += scratch[turn][i].y; }
    turn ^= 1u;
    return s;
}
__device__ __forceinline__ float group_sum(float v, float2 (*scratch)[32], uint32_t& turn) {
    v = warp_sum(v);
    if (blockDim.x == 32) return v;
    const uint32_t warps = blockDim.x / 32;
    if ((threadIdx.x & 31) == 0) scratch[turn][threadIdx.x >> 5].x = v;
    __syncthreads();
    float s = scratch[turn][0].x;
    for (uint32_t i = 1; i < warps; ++i) s += scratch[turn][i].x;
    turn ^= 1u;
    return s;
}

// blockDim = (G, groups in the block). HOLD: gamma and beta stay in registers and the next row is loaded ahead.
template <typename T, typename W, int VB, int NV, bool HOLD, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_forward_kernel(NormArgs a) {
    using V = Pack<T, VB>;
    constexpr int N = V::N;
    __shared__ float2 scratch[2][32];
    uint32_t turn = 0;
    const uint32_t G = blockDim.x, vecs = a.H / N;
    const W* gamma = static_cast<const W*>(a.gamma);
    const W* beta = static_cast<const W*>(a.beta);
    const float inv = 1.f / (float)a.H;
    const uint64_t step = (uint64_t)gridDim.x * blockDim.y;
    uint64_t r = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y;
    V next[NV];
    float g[HOLD ? NV * N : N], b[HOLD ? NV * N : N];
    const auto fetch = [&](uint64_t row) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = i * G + threadIdx.x;
            if (q < vecs) next[i].load(x + q * N); else next[i].clear();
        }
    };
    if (r < a.rows) fetch(r);
    if (HOLD) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = i * G + threadIdx.x;
            if (q < vecs) { load_weights<W, N>(g + i * N, gamma, q * N, 1.f); load_weights<W, N>(b + i * N, beta, q * N, 0.f); }
        }
    }
    for (; r < a.rows; r += step) {
        V x[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = next[i];
        if (HOLD && r + step < a.rows) fetch(r + step);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) s += x[i].get(j);
        const float mean = group_sum(s, scratch, turn) * inv;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * G + threadIdx.x < vecs) {
#pragma unroll
                for (int j = 0; j < N; ++j) { const float d = x[i].get(j) - mean; s = fmaf(d, d, s); }
            }
        const float rstd = 1.f / sqrtf(group_sum(s, scratch, turn) * inv + a.eps);
        T* y = static_cast<T*>(a.y) + r * a.y_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = i * G + threadIdx.x;
            if (q < vecs) {
                if (!HOLD) { load_weights<W, N>(g, gamma, q * N, 1.f); load_weights<W, N>(b, beta, q * N, 0.f); }
                float o[N];
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] = fmaf((x[i].get(j) - mean) * rstd, g[HOLD ? i * N + j : j], b[HOLD ? i * N + j : j]);
                V::store(y + q * N, o);
            }
        }
        if (threadIdx.x == 0) {
            if (a.mean_out) a.mean_out[r] = mean;
            if (a.rstd_out) a.rstd_out[r] = rstd;
        }
        if (!HOLD && r + step < a.rows) fetch(r + step);
    }
}

// blockDim = (G, groups in the block); a group of threads walks the rows of one RowWalk. AHEAD: the next row is loaded ahead.
template <typename T, typename W, int VB, int NV, bool AHEAD, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_backward_kernel(NormArgs a) {
    using V = Pack<T, VB>;
    constexpr int N = V::N, E = NV * N;
    __shared__ float2 scratch[2][32];
    uint32_t turn = 0;
    const uint32_t G = blockDim.x, vecs = a.H / N, group = blockIdx.x * blockDim.y + threadIdx.y;
    if (group >= a.groups) return;                                   // whole groups; a group of several warps is a whole block
    RowWalk walk(a, group);
    const float inv = 1.f / (float)a.H;
    V nx[NV], ny[NV];
    float nmean = 0.f, nrstd = 0.f;
    const auto fetch = [&](uint64_t row) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = i * G + threadIdx.x;
            if (q < vecs) { nx[i].load(x + q * N); ny[i].load(dy + q * N); }
            else { nx[i].clear(); ny[i].clear(); }                   // dy = 0: adds nothing to any sum
        }
        nmean = a.mean[row]; nrstd = a.rstd[row];
    };
    float g[E], dg[E], db[E];
    if (walk.r0 < walk.r1) fetch(walk.r0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t q = i * G + threadIdx.x;
#pragma unroll
        for (int j = 0; j < N; ++j) g[i * N + j] = dg[i * N + j] = db[i * N + j] = 0.f;
        if (q < vecs) load_weights<W, N>(g + i * N, static_cast<const W*>(a.gamma), q * N, 1.f);
    }
    const auto leave = [&]() {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = i * G + threadIdx.x;
            if (q < vecs) store_slot<N>(a, walk.slot(), q * N, dg + i * N, db + i * N);
        }
    };
    for (uint64_t r = walk.r0; r < walk.r1; ++r) {
        V x[NV], dy[NV];
        const float mean = nmean, rstd = nrstd;
#pragma unroll
        for (int i = 0; i < NV; ++i) { x[i] = nx[i]; dy[i] = ny[i]; }
        if (AHEAD && r + 1 < walk.r1) fetch(r + 1);
        float2 s = make_float2(0.f, 0.f);
        if (a.slots && walk.leaves(r)) {
            if (walk.any) leave();
#pragma unroll
            for (int j = 0; j < E; ++j) dg[j] = db[j] = 0.f;
            walk.go_to(r);
        }
        const bool counts = a.slots && walk.counts(r);
        walk.any |= counts;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float d = dy[i].get(j), xh = (x[i].get(j) - mean) * rstd, u = d * g[i * N + j];
                s.x += u;
                s.y = fmaf(u, xh, s.y);
                if (counts) { dg[i * N + j] = fmaf(d, xh, dg[i * N + j]); db[i * N + j] += d; }
            }
        if (a.dx) {
            s = group_sum(s, scratch, turn);
            const float c1 = s.x * inv, c2 = s.y * inv;
            T* dx = static_cast<T*>(a.dx) + r * a.dx_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t q = i * G + threadIdx.x;
                if (q < vecs) {
                    float o[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float xh = (x[i].get(j) - mean) * rstd;
                        o[j] = rstd * (fmaf(dy[i].get(j), g[i * N + j], -c1) - xh * c2);
                    }
                    V::store(dx + q * N, o);
                }
            }
        }
        if (!AHEAD && r + 1 < walk.r1) fetch(r + 1);
    }
    if (a.slots && walk.any) leave();
}

// Threads for a row of `vecs` vectors, NV each, and rows of a block of 128 threads where a warp is enough for one.
static inline dim3 group_shape(uint32_t vecs, uint32_t nv) {
    const uint32_t g = ((vecs + nv - 1) / nv + 31) / 32 * 32;
    return dim3(g, g == 32 ? 4 : 1);
}

template <typename T, typename W, int VB, int NV, bool HOLD, int MAXT>
static cudaError_t forward_run(const NormArgs& a, int sms, cudaStream_t st) {
    const dim3 block = group_shape(a.H / (VB / (uint32_t)sizeof(T)), NV);
    const uint64_t blocks = (a.rows + block.y - 1) / block.y, cap = (uint64_t)sms * (MAXT == 1024 ? 1024 : 768) / (block.x * block.y);
    norm_forward_kernel<T, W, VB, NV, HOLD, MAXT><<<(uint32_t)(blocks < cap ? blocks : cap ? cap : 1), block, 0, st>>>(a);
    return cudaGetLastError();
}

// cudaErrorNotSupported: the row does not fit.
template <typename T, typename W> static cudaError_t forward_rows(const NormArgs& a, uint32_t v, int sms, cudaStream_t st) {
    const uint32_t vecs = a.H * (uint32_t)sizeof(T) / v;
    if (v == 16) {
        constexpr int most = sizeof(T) == 2 ? 2 : 4;
        if (vecs <= 256) return forward_run<T, W, 16, 1, true, 512>(a, sms, st);
        if (vecs <= 512 * most) return forward_run<T, W, 16, most, true, 512>(a, sms, st);
        if (vecs <= 8192) return forward_run<T, W, 16, 8, false, 1024>(a, sms, st);
        return cudaErrorNotSupported;
    }
    constexpr int E = sizeof(T);
    if constexpr (E == 2) if (v == 4) {
        if (vecs <= 2048) return forward_run<T, W, 4, 4, true, 512>(a, sms, st);
        if (vecs <= 16384) return forward_run<T, W, 4, 16, false, 1024>(a, sms, st);
        return cudaErrorNotSupported;
    }
    if (vecs <= 2048) return forward_run<T, W, E, 4, true, 512>(a, sms, st);
    if (vecs <= 16384) return forward_run<T, W, E, 16, false, 1024>(a, sms, st);
    return cudaErrorNotSupported;
}

template <typename T, typename W, int VB, int NV>
static cudaError_t backward_run(const NormArgs& a, cudaStream_t st) {
    const dim3 block = group_shape(a.H / (VB / (uint32_t)sizeof(T)), NV);
    norm_backward_kernel<T, W, VB, NV, NV * Pack<T, VB>::WORDS <= 8, 512><<<(a.groups + block.y - 1) / block.y, block, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T, typename W> static cudaError_t backward_rows(const NormArgs& a, uint32_t v, cudaStream_t st) {
    const uint32_t vecs = a.H * (uint32_t)sizeof(T) / v;
    if (v == 16) {
        if (vecs <= 256) return backward_run<T, W, 16, 1>(a, st);
        if (vecs <= 1024) return backward_run<T, W, 16, 2>(a, st);
        if constexpr (sizeof(T) == 4) { if (vecs <= 2048) return backward_run<T, W, 16, 4>(a, st); }
        return cudaErrorNotSupported;
    }
    constexpr int E = sizeof(T);
    if constexpr (E == 2) if (v == 4) {
        if (vecs <= 2048) return backward_run<T, W, 4, 4>(a, st);
        if (vecs <= 4096) return backward_run<T, W, 4, 8>(a, st);
        return cudaErrorNotSupported;
    }
    if (vecs <= 2048) return backward_run<T, W, E, 4>(a, st);
    if (vecs <= 8192) return backward_run<T, W, E, 16>(a, st);
    return cudaErrorNotSupported;
}

}  // namespace ftc
