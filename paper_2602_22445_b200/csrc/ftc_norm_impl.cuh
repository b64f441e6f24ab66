// Layer norm on rows that fit the registers of a thread block.
//
// A group of G threads (a warp, or a block of up to 512) holds a row, 16 elements a thread: vector i of thread t is vector i*G + t of
// the row, so every load and store of a warp is one contiguous run. Statistics are taken in two steps from the registers (mean, then
// squared distances), which no common offset of the row can spoil. A group walks many rows with gamma, beta and the column sums in registers.
//
// Rows come in through a ring of D rows in shared memory, filled by asynchronous copies (16 or 4 bytes a thread) that run D - 1 rows
// ahead: what an SM has under way no longer depends on registers. Each thread copies what it reads itself, so the ring needs no barrier. The
// exception is 16-bit rows that begin between two 4-byte words (ODD: an odd H or stride): their words are copied whole, and a thread
// shifts its pair of elements out of two neighbouring words, which takes one barrier a row. The word that reaches over the
// first row's beginning or the last row's end is put together from its one element.
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

// Sums over the group. With more than one warp they go through shared memory; `turn` alternates between two places, so that one
// barrier a call is enough (a place is written again only behind the barrier of the call in between). Places of warps that do not
// exist hold zeros.
constexpr int kMaxGroup = 512, kMaxWarps = kMaxGroup / 32;
struct Scratch { float4 pair[2][kMaxWarps / 2]; };

__device__ __forceinline__ void clear_scratch(Scratch& s) {
    const uint32_t t = threadIdx.y * blockDim.x + threadIdx.x;
    if (t < kMaxWarps) (&s.pair[0][0])[t] = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncthreads();
}
__device__ __forceinline__ float2 group_sum(float2 v, Scratch& scratch, uint32_t& turn) {
#pragma unroll
    for (int o = 16; o; o >>= 1) { v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o); v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o); }
    if (blockDim.x == 32) return v;
    float4* place = scratch.pair[turn];
    if ((threadIdx.x & 31) == 0) reinterpret_cast<float2*>(place)[threadIdx.x >> 5] = v;
    __syncthreads();
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kMaxWarps / 2; ++i) { const float4 q = place[i]; s.x += q.x + q.z; s.y += q.y + q.w; }
    turn ^= 1u;
    return s;
}
__device__ __forceinline__ float group_sum(float v, Scratch& scratch, uint32_t& turn) {
    v = warp_sum(v);
    if (blockDim.x == 32) return v;
    float4* place = scratch.pair[turn];
    if ((threadIdx.x & 31) == 0) reinterpret_cast<float*>(place)[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxWarps / 4; ++i) { const float4 q = place[i]; s += (q.x + q.y) + (q.z + q.w); }
    turn ^= 1u;
    return s;
}
__device__ __forceinline__ void group_barrier() { if (blockDim.x == 32) __syncwarp(); else __syncthreads(); }

template <int VB> __device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
    if constexpr (VB == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_batch() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(PENDING) : "memory"); }

// The rows of one array in the ring: NV vectors of VB bytes for each thread, n elements in a row, `rows` rows.
template <typename T, int VB, int NV, bool ODD> struct RingRows {
    static constexpr int N = VB / (int)sizeof(T);
    const T* base;
    uint64_t stride, rows;
    uint32_t n, vecs;
    // Bytes that one row takes up in the ring.
    static __host__ __device__ uint32_t bytes(uint32_t G) { return NV * G * VB + (ODD ? 16 : 0); }
    __device__ __forceinline__ uint32_t odd(uint64_t r) const { return ODD ? (uint32_t)(reinterpret_cast<uintptr_t>(base + r * stride) >> 1) & 1u : 0u; }
    __device__ __forceinline__ void fetch(char* place, uint64_t r) const {
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(place);
        if constexpr (!ODD) {
            const T* p = base + r * stride;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t q = i * blockDim.x + threadIdx.x;
                if (q < vecs) copy_async<VB>(dst + q * VB, p + q * N);
            }
        } else {
            const uint32_t s = odd(r), words = (s + n + 1) / 2;
            const T* p = base + r * stride - s;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t q = i * blockDim.x + threadIdx.x;
                if (q >= words) continue;
                if (q == 0 && s && r == 0) reinterpret_cast<uint32_t*>(place)[0] = (uint32_t)reinterpret_cast<const uint16_t*>(p)[1] << 16;
                else if (q == words - 1 && ((s + n) & 1u) && r + 1 == rows) reinterpret_cast<uint32_t*>(place)[q] = reinterpret_cast<const uint16_t*>(p)[2 * q];
                else copy_async<4>(dst + q * 4, p + q * 2);
            }
        }
    }
    // Vector i of this thread; zeros behind the row's end.
    __device__ __forceinline__ void read(Pack<T, VB>& v, const char* place, int i, uint32_t s) const {
        const uint32_t q = i * blockDim.x + threadIdx.x;
        if (q >= vecs) { v.clear(); return; }
        if constexpr (VB == 16) { const uint4 w = reinterpret_cast<const uint4*>(place)[q]; v.r[0] = w.x; v.r[1] = w.y; v.r[2] = w.z; v.r[3] = w.w; }
        else if constexpr (!ODD) v.r[0] = reinterpret_cast<const uint32_t*>(place)[q];
        else {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(place) + q;
            v.r[0] = s ? __funnelshift_r(w[0], w[1], 16) : w[0];
            if (2 * q + 1 >= n) v.r[0] &= 0xFFFFu;                   // an odd row's last element stands alone
        }
    }
};

// A vector of results to column c of a row (ODD: a pair that may begin between words, or be one element).
template <typename T, int VB, bool ODD> __device__ __forceinline__ void store_vector(T* row, uint32_t c, uint32_t n, const float* v) {
    if constexpr (!ODD) Pack<T, VB>::store(row + c, v);
    else {
        if (c + 1 < n && (reinterpret_cast<uintptr_t>(row) & 3u) == 0) { Pack<T, 4>::store(row + c, v); return; }
        row[c] = from_f32<T>(v[0]);
        if (c + 1 < n) row[c + 1] = from_f32<T>(v[1]);
    }
}

// Weights of a thread's vector; ODD: of a pair of which the second may not exist.
template <typename W, int N, bool ODD> __device__ __forceinline__ void vector_weights(float* v, const W* w, uint32_t c, uint32_t n, float other) {
    if constexpr (!ODD) load_weights<W, N>(v, w, c, other);
    else { v[0] = w ? to_f32(w[c]) : other; v[1] = w && c + 1 < n ? to_f32(w[c + 1]) : other; }
}

// blockDim = (G, groups in the block).
template <typename T, typename W, int VB, int NV, bool ODD, int D>
__global__ void __launch_bounds__(kMaxGroup) norm_forward_kernel(NormArgs a) {
    using V = Pack<T, VB>;
    using Rows = RingRows<T, VB, NV, ODD>;
    constexpr int N = V::N;
    extern __shared__ uint4 ring_memory[];
    __shared__ Scratch scratch;
    uint32_t turn = 0;
    const uint32_t G = blockDim.x, vecs = (a.H + N - 1) / N, bytes = Rows::bytes(G);
    char* ring = reinterpret_cast<char*>(ring_memory) + threadIdx.y * D * bytes;
    const Rows in{static_cast<const T*>(a.x), a.x_stride, a.rows, a.H, vecs};
    const float inv = 1.f / (float)a.H;
    const uint64_t step = (uint64_t)gridDim.x * blockDim.y;
    uint64_t r = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y;
#pragma unroll
    for (int d = 0; d < D - 1; ++d) {
        if (r + d * step < a.rows) in.fetch(ring + d * bytes, r + d * step);
        copies_end_batch();
    }
    float g[NV * N], b[NV * N];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t q = i * G + threadIdx.x;
        if (q < vecs) {
            vector_weights<W, N, ODD>(g + i * N, static_cast<const W*>(a.gamma), q * N, a.H, 1.f);
            vector_weights<W, N, ODD>(b + i * N, static_cast<const W*>(a.beta), q * N, a.H, 0.f);
        }
    }
    clear_scratch(scratch);
    uint32_t stage = 0;
    for (; r < a.rows; r += step) {
        copies_wait<D - 2>();
        if (ODD) group_barrier();
        V x[NV];
        const uint32_t s0 = in.odd(r);
#pragma unroll
        for (int i = 0; i < NV; ++i) in.read(x[i], ring + stage * bytes, i, s0);
        const uint32_t last = stage == 0 ? D - 1 : stage - 1;
        if (r + (D - 1) * step < a.rows) in.fetch(ring + last * bytes, r + (D - 1) * step);
        copies_end_batch();
        stage = stage + 1 == D ? 0 : stage + 1;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) s += x[i].get(j);
        const float mean = group_sum(s, scratch, turn) * inv;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float d = x[i].get(j) - mean;
                const uint32_t c = (i * G + threadIdx.x) * N + (ODD ? j : 0);
                if (c < a.H) s = fmaf(d, d, s);
            }
        const float rstd = 1.f / sqrtf(group_sum(s, scratch, turn) * inv + a.eps);
        T* y = static_cast<T*>(a.y) + r * a.y_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = i * G + threadIdx.x;
            if (q < vecs) {
                float o[N];
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] = fmaf((x[i].get(j) - mean) * rstd, g[i * N + j], b[i * N + j]);
                store_vector<T, VB, ODD>(y, q * N, a.H, o);
            }
        }
        if (threadIdx.x == 0) {
            if (a.mean_out) a.mean_out[r] = mean;
            if (a.rstd_out) a.rstd_out[r] = rstd;
        }
    }
}

// blockDim = (G, groups in the block); a group of threads walks the rows of one RowWalk.
template <typename T, typename W, int VB, int NV, bool ODD, int D>
__global__ void __launch_bounds__(kMaxGroup) norm_backward_kernel(NormArgs a) {
    using V = Pack<T, VB>;
    using Rows = RingRows<T, VB, NV, ODD>;
    constexpr int N = V::N, E = NV * N;
    extern __shared__ uint4 ring_memory[];
    __shared__ Scratch scratch;
    uint32_t turn = 0;
    const uint32_t G = blockDim.x, vecs = (a.H + N - 1) / N, bytes = Rows::bytes(G), group = blockIdx.x * blockDim.y + threadIdx.y;
    char* ring = reinterpret_cast<char*>(ring_memory) + threadIdx.y * D * 2 * bytes;
    const Rows xs{static_cast<const T*>(a.x), a.x_stride, a.rows, a.H, vecs}, ys{static_cast<const T*>(a.dy), a.dy_stride, a.rows, a.H, vecs};
    clear_scratch(scratch);
    if (group >= a.groups) return;                                   // whole warps, and in blocks of one group nobody
    RowWalk walk(a, group);
    const float inv = 1.f / (float)a.H;
#pragma unroll
    for (int d = 0; d < D - 1; ++d) {
        if (walk.r0 + d < walk.r1) { xs.fetch(ring + 2 * d * bytes, walk.r0 + d); ys.fetch(ring + (2 * d + 1) * bytes, walk.r0 + d); }
        copies_end_batch();
    }
    float g[E], dg[E], db[E];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t q = i * G + threadIdx.x;
#pragma unroll
        for (int j = 0; j < N; ++j) g[i * N + j] = dg[i * N + j] = db[i * N + j] = 0.f;
        if (q < vecs) vector_weights<W, N, ODD>(g + i * N, static_cast<const W*>(a.gamma), q * N, a.H, 1.f);
    }
    const auto leave = [&]() {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = i * G + threadIdx.x;
            if (q >= vecs) continue;
            if constexpr (!ODD) store_slot<N>(a, walk.slot(), q * N, dg + i * N, db + i * N);
            else {
                store_slot<1>(a, walk.slot(), q * 2, dg + i * N, db + i * N);
                if (q * 2 + 1 < a.H) store_slot<1>(a, walk.slot(), q * 2 + 1, dg + i * N + 1, db + i * N + 1);
            }
        }
    };
    float nmean = 0.f, nrstd = 0.f;
    if (walk.r0 < walk.r1) { nmean = a.mean[walk.r0]; nrstd = a.rstd[walk.r0]; }
    uint32_t stage = 0;
    for (uint64_t r = walk.r0; r < walk.r1; ++r) {
        copies_wait<D - 2>();
        if (ODD) group_barrier();
        V x[NV], dy[NV];
        const uint32_t sx = xs.odd(r), sy = ys.odd(r);
#pragma unroll
        for (int i = 0; i < NV; ++i) { xs.read(x[i], ring + 2 * stage * bytes, i, sx); ys.read(dy[i], ring + (2 * stage + 1) * bytes, i, sy); }
        const uint32_t last = stage == 0 ? D - 1 : stage - 1;
        if (r + (D - 1) < walk.r1) { xs.fetch(ring + 2 * last * bytes, r + (D - 1)); ys.fetch(ring + (2 * last + 1) * bytes, r + (D - 1)); }
        copies_end_batch();
        stage = stage + 1 == D ? 0 : stage + 1;
        const float mean = nmean, rstd = nrstd;
        if (r + 1 < walk.r1) { nmean = a.mean[r + 1]; nrstd = a.rstd[r + 1]; }
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
            for (int j = 0; j < N; ++j) {                            // behind the row's end dy = 0 adds nothing
                const float d = dy[i].get(j), xh = (x[i].get(j) - mean) * rstd, u = d * g[i * N + j];
                s.x += u;
                s.y = fmaf(u, xh, s.y);
                if (counts) { dg[i * N + j] = fmaf(d, xh, dg[i * N + j]); db[i * N + j] += d; }
            }
        if (!a.dx) continue;
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
                store_vector<T, VB, ODD>(dx, q * N, a.H, o);
            }
        }
    }
    if (a.slots && walk.any) leave();
}

// Threads that hold a row of H elements, 16 each, and rows of a block of 128 threads where a warp is enough for one.
static inline uint32_t group_threads(uint32_t H) { return (H / 16 + 1 + 31) / 32 * 32; }
static inline dim3 group_shape(uint32_t vecs, uint32_t nv) {
    const uint32_t g = ((vecs + nv - 1) / nv + 31) / 32 * 32;
    return dim3(g, g == 32 ? 4 : 1);
}

template <typename K> static cudaError_t allow_shared(K kernel, size_t bytes) {
    return bytes <= 40 * 1024 ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T, typename W, int VB, int NV, bool ODD, int D> static cudaError_t forward_run(const NormArgs& a, int sms, cudaStream_t st) {
    constexpr uint32_t N = VB / (uint32_t)sizeof(T);
    const dim3 block = group_shape((a.H + N - 1) / N + (ODD ? 1 : 0), NV);
    const size_t smem = (size_t)block.y * D * RingRows<T, VB, NV, ODD>::bytes(block.x);
    const cudaError_t e = allow_shared(norm_forward_kernel<T, W, VB, NV, ODD, D>, smem);
    if (e != cudaSuccess) return e;
    const uint64_t blocks = (a.rows + block.y - 1) / block.y, cap = (uint64_t)sms * (768 / (block.x * block.y) ? 768 / (block.x * block.y) : 1);
    norm_forward_kernel<T, W, VB, NV, ODD, D><<<(uint32_t)(blocks < cap ? blocks : cap), block, smem, st>>>(a);
    return cudaGetLastError();
}

// cudaErrorNotSupported: the row does not fit.
template <typename T, typename W> static cudaError_t forward_rows(const NormArgs& a, uint32_t v, int sms, cudaStream_t st) {
    constexpr int E = sizeof(T), D = E == 2 ? 4 : 3;
    if (a.H > 16 * kMaxGroup || (v == 2 && a.H > 16 * kMaxGroup - 2)) return cudaErrorNotSupported;
    if (v == 16) return a.H <= 32 * 16 / E ? forward_run<T, W, 16, 1, false, D>(a, sms, st) : forward_run<T, W, 16, E, false, D>(a, sms, st);
    if constexpr (E == 4) return forward_run<T, W, 4, 16, false, D>(a, sms, st);
    else return v == 4 ? forward_run<T, W, 4, 8, false, D>(a, sms, st) : forward_run<T, W, 4, 8, true, D>(a, sms, st);
}

template <typename T, typename W, int VB, int NV, bool ODD, int D> static cudaError_t backward_run(const NormArgs& a, cudaStream_t st) {
    constexpr uint32_t N = VB / (uint32_t)sizeof(T);
    const dim3 block = group_shape((a.H + N - 1) / N + (ODD ? 1 : 0), NV);
    const size_t smem = (size_t)block.y * D * 2 * RingRows<T, VB, NV, ODD>::bytes(block.x);
    const cudaError_t e = allow_shared(norm_backward_kernel<T, W, VB, NV, ODD, D>, smem);
    if (e != cudaSuccess) return e;
    norm_backward_kernel<T, W, VB, NV, ODD, D><<<(a.groups + block.y - 1) / block.y, block, smem, st>>>(a);
    return cudaGetLastError();
}

template <typename T, typename W> static cudaError_t backward_rows(const NormArgs& a, uint32_t v, cudaStream_t st) {
    constexpr int E = sizeof(T), D = E == 2 ? 3 : 2;
    if (a.H > 16 * kMaxGroup || (v == 2 && a.H > 16 * kMaxGroup - 2)) return cudaErrorNotSupported;
    if (v == 16) return a.H <= 32 * 16 / E ? backward_run<T, W, 16, 1, false, D>(a, st) : backward_run<T, W, 16, E, false, D>(a, st);
    if constexpr (E == 4) return backward_run<T, W, 4, 16, false, D>(a, st);
    else return v == 4 ? backward_run<T, W, 4, 8, false, D>(a, st) : backward_run<T, W, 4, 8, true, D>(a, st);
}

}  // namespace ftc
