// Layer norm forward and backward, with the weight gradients of each process of a data-parallel job: choice of kernels, and the
// kernels for rows that do not fit the registers of a thread block (the others: ftc_norm_impl.cuh).
//
// Weight gradients are sums over rows: a group of threads walks the rows [b*R, (b+1)*R) in order and keeps one partial sum per column,
// which it leaves in the workspace whenever the row's process changes and at its end. Group b and process p share slot b + p: going on
// by one row either the group or the process grows, so no two (group, process) pairs that have rows in common meet in one slot, and
// groups + P slots are enough however the rows are divided. A second kernel adds the slots of each process in ascending order and lays
// the sums out as messages.
#include "ftc_norm_impl.cuh"

namespace ftc {

constexpr uint32_t kThreads = 256;

__device__ __forceinline__ double block_sum(double v, double* scratch) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0;
    for (uint32_t i = 0; i < kThreads / 32; ++i) s += scratch[i];
    return s;
}

// Rows of up to 32 elements a thread, from memory to registers and back; weights come from the caches. For rows that a group of 16
// elements a thread does not hold (8192 < H <= 32768); bound by the chain of one row (bf16, 40 rows of 11720: 4 us; walking the row three
// times took 27).
constexpr int kLongest = 32 * 1024;
template <typename T, typename W, int VB>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(NormArgs a) {
    using V = Pack<T, VB>;
    constexpr int N = V::N, NV = 32 / N;
    __shared__ float scratch[2][32];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x / 32, v0 = warp * 32 * NV + lane, vecs = a.H / N;
    const auto sum = [&](float v, int turn) {
        v = warp_sum(v);
        if (lane == 0) scratch[turn][warp] = v;
        __syncthreads();
        return warp_sum(lane < warps ? scratch[turn][lane] : 0.f);
    };
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        T* y = static_cast<T*>(a.y) + r * a.y_stride;
        V v[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (v0 + i * 32 < vecs) v[i].load(x + (v0 + i * 32) * N); else v[i].clear();
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) s += v[i].get(j);
        const float mean = sum(s, 0) / a.H;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (v0 + i * 32 < vecs) {
#pragma unroll
                for (int j = 0; j < N; ++j) { const float d = v[i].get(j) - mean; s = fmaf(d, d, s); }
            }
        const float rstd = inverse_root(sum(s, 1) / a.H + a.eps);    // each place is written again behind the other one's barrier
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t c = (v0 + i * 32) * N;
            if (c >= a.H) continue;
            float g[N], b[N], o[N];
            load_weights<W, N>(g, static_cast<const W*>(a.gamma), c, 1.f);
            load_weights<W, N>(b, static_cast<const W*>(a.beta), c, 0.f);
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = fmaf((v[i].get(j) - mean) * rstd, g[j], b[j]);
            V::store(y + c, o);
        }
        if (threadIdx.x == 0) {
            if (a.mean_out) a.mean_out[r] = mean;
            if (a.rstd_out) a.rstd_out[r] = rstd;
        }
    }
}

// Wider still: a block walks a row three times; rows come back from the caches. A thread adds 64 numbers in float32 and such sums in float64: a
// row of 2^24 numbers around 100 has its mean within 1e-5 (in float32 throughout 0.08).
template <typename V> __device__ __forceinline__ double long_sum(uint32_t n, double* scratch, V value) {
    double s = 0;
    uint32_t h = threadIdx.x;
    for (; h + 63 * kThreads < n; h += 64 * kThreads) {
        float part = 0.f;
#pragma unroll 1
        for (uint32_t g = h; g < h + 64 * kThreads; g += 16 * kThreads) {
            float v[16];                                             // all loads out at once
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = value(g + i * kThreads);
#pragma unroll
            for (int i = 0; i < 16; ++i) part += v[i];
        }
        s += part;
    }
    float part = 0.f;
#pragma unroll 4
    for (; h < n; h += kThreads) part += value(h);
    s += part;
    return block_sum(s, scratch);
}
template <typename T, typename W>
__global__ void __launch_bounds__(kThreads) norm_forward_long_kernel(NormArgs a) {
    __shared__ double scratch[kThreads / 32];
    const W* gamma = static_cast<const W*>(a.gamma);
    const W* beta = static_cast<const W*>(a.beta);
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        T* y = static_cast<T*>(a.y) + r * a.y_stride;
        const float mean = (float)(long_sum(a.H, scratch, [&](uint32_t h) { return to_f32(x[h]); }) / a.H);
        const double squares = long_sum(a.H, scratch, [&](uint32_t h) { const float d = to_f32(x[h]) - mean; return d * d; });
        const float rstd = 1.f / sqrtf((float)(squares / a.H) + a.eps);
        for (uint32_t h = threadIdx.x; h < a.H; h += 8 * kThreads) {     // eight numbers' loads before the first store, which might write to x
            float v[8], g[8], b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = h + i * kThreads;
                v[i] = g[i] = b[i] = 0.f;
                if (c < a.H) { v[i] = to_f32(x[c]); g[i] = gamma ? to_f32(gamma[c]) : 1.f; b[i] = beta ? to_f32(beta[c]) : 0.f; }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (h + i * kThreads < a.H) y[h + i * kThreads] = from_f32<T>((v[i] - mean) * rstd * g[i] + b[i]);
        }
        if (threadIdx.x == 0) {
            if (a.mean_out) a.mean_out[r] = mean;
            if (a.rstd_out) a.rstd_out[r] = rstd;
        }
    }
}

// dx alone, for H > 8192 (f16, 6534 rows of 13256 over 955 processes: columns 78 us, dx 111, messages 46; one kernel for columns and dx
// would save reading 346 MB again. No block holds the column sums of such a row; a cluster of blocks that exchange a row's two sums would). KEEP: the row stays in registers, four vectors a thread, as loaded; else a block walks it twice, the second time from the
// caches.
template <typename T, typename W, int VB, bool KEEP>
__global__ void __launch_bounds__(1024) norm_backward_long_kernel(NormArgs a) {
    using V = Pack<T, VB>;
    constexpr int N = V::N, NV = KEEP ? 4 : 1;
    __shared__ float2 scratch[32];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x / 32, step = blockDim.x * N;
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + r * a.dy_stride;
        T* dx = static_cast<T*>(a.dx) + r * a.dx_stride;
        const float mean = a.mean[r], rstd = a.rstd[r];
        V v[NV], d[NV];
        float s1 = 0.f, s2 = 0.f;
        const auto add = [&](const V& vi, const V& di, uint32_t c) {
            float g[N];
            load_weights<W, N>(g, static_cast<const W*>(a.gamma), c, 1.f);
#pragma unroll
            for (int j = 0; j < N; ++j) { const float u = di.get(j) * g[j]; s1 += u; s2 = fmaf(u, (vi.get(j) - mean) * rstd, s2); }
        };
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t c = threadIdx.x * N + i * step;
                if (c < a.H) { v[i].load(x + c); d[i].load(dy + c); }            // N divides H
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t c = threadIdx.x * N + i * step;
                if (c < a.H) add(v[i], d[i], c);
            }
        } else {
#pragma unroll 4
            for (uint32_t c = threadIdx.x * N; c < a.H; c += step) { v[0].load(x + c); d[0].load(dy + c); add(v[0], d[0], c); }
        }
        s1 = warp_sum(s1); s2 = warp_sum(s2);
        __syncthreads();
        if (lane == 0) scratch[warp] = make_float2(s1, s2);
        __syncthreads();
        const float2 part = lane < warps ? scratch[lane] : make_float2(0.f, 0.f);
        const float c1 = warp_sum(part.x) / a.H, c2 = warp_sum(part.y) / a.H;
        const auto give = [&](const V& vi, const V& di, uint32_t c) {
            float g[N], o[N];
            load_weights<W, N>(g, static_cast<const W*>(a.gamma), c, 1.f);
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = rstd * (fmaf(di.get(j), g[j], -c1) - (vi.get(j) - mean) * rstd * c2);
            V::store(dx + c, o);
        };
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t c = threadIdx.x * N + i * step;
                if (c < a.H) give(v[i], d[i], c);
            }
        } else {
#pragma unroll 4
            for (uint32_t c = threadIdx.x * N; c < a.H; c += step) { v[0].load(x + c); d[0].load(dy + c); give(v[0], d[0], c); }
        }
    }
}

// The weight gradients alone (H > 8192): a thread owns N neighbouring columns and walks its group's rows, four rows' loads out at once. No
// sum over a row is needed.
template <typename T, int VB>
__global__ void __launch_bounds__(kThreads) norm_columns_kernel(NormArgs a) {
    constexpr int N = VB / (int)sizeof(T), AHEAD = 4;
    using V = Pack<T, VB>;
    const uint32_t own = (blockIdx.x * kThreads + threadIdx.x) * N, c = own < a.H ? own : a.H - N;         // N divides H
    later_kernel_may_start();
    RowWalk walk(a, blockIdx.y);
    walk.find();
    if (__all_sync(0xFFFFFFFFu, own >= a.H)) return;                 // warps stay whole for the walk
    float dg[N] = {}, db[N] = {};
    for (uint32_t r = walk.r0; r < walk.r1; r += AHEAD) {                // r1 + AHEAD stays below 2^32
        V x[AHEAD], dy[AHEAD];
        float mean[AHEAD], rstd[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (r + i < walk.r1) {
                x[i].load(static_cast<const T*>(a.x) + (uint64_t)(r + i) * a.x_stride + c);
                dy[i].load(static_cast<const T*>(a.dy) + (uint64_t)(r + i) * a.dy_stride + c);
                mean[i] = a.mean[r + i]; rstd[i] = a.rstd[r + i];
            }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (r + i < walk.r1) {
                if (walk.leaves(r + i)) {
                    if (walk.any && own < a.H) store_slot<N>(a, walk.slot(), c, dg, db);
                    walk.go_to(r + i);
#pragma unroll
                    for (int j = 0; j < N; ++j) dg[j] = db[j] = 0.f;
                }
                if (walk.counts(r + i)) {
                    walk.any = true;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float g = dy[i].get(j);
                        dg[j] = fmaf(g, (x[i].get(j) - mean[i]) * rstd[i], dg[j]);
                        db[j] += g;
                    }
                }
            }
    }
    if (walk.any && own < a.H) store_slot<N>(a, walk.slot(), c, dg, db);
}

// dgamma[s][p][e], dbeta[s][p][e] from the slots: Q warps add the slots of one process for C columns a lane, each every Q-th slot, and
// their sums are added in order.
template <int Q, int C>
__global__ void __launch_bounds__(Q == 32 ? 1024 : 256) norm_messages_kernel(NormArgs a, uint32_t tiles, uint32_t items) {
    constexpr int WARPS = Q == 32 ? 32 : 8;
    __shared__ float part[2][WARPS][32];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, turn = warp % Q, item = blockIdx.x * (WARPS / Q) + warp / Q;
    const uint32_t p = item / tiles, h0 = (item - p * tiles) * (32 * C) + lane, S = (a.H + a.k - 1) / a.k;
    float g[C] = {}, b[C] = {};
    const bool wanted = item < items && h0 < a.H;
    const uint32_t lo = wanted ? first_row(a, p) : 0, hi = wanted ? first_row(a, p + 1) : 0;
    wait_for_earlier_kernel();
    if (lo < hi) {
        const uint32_t last = (hi - 1) / a.rows_per_group;
#pragma unroll(C > 1 ? 1 : 4)
        for (uint32_t grp = lo / a.rows_per_group + turn; grp <= last; grp += Q) {
            const float* slot = a.slots + ((uint64_t)grp + p) * 2 * a.H + h0;
#pragma unroll
            for (int i = 0; i < C; ++i)
                if (i == 0 || h0 + i * 32 < a.H) { g[i] += slot[i * 32]; b[i] += slot[a.H + i * 32]; }
        }
    }
    if (Q > 1) {                                                     // C = 1
        part[0][warp][lane] = g[0]; part[1][warp][lane] = b[0];
        __syncthreads();
        if (turn) return;
        for (int i = 1; i < Q; ++i) { g[0] += part[0][warp + i][lane]; b[0] += part[1][warp + i][lane]; }
    }
    if (item >= items) return;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const uint32_t h = h0 + i * 32, s = h / a.k;
        if (s >= S) return;                                          // h beyond H: the last message's fill, zeros
        const uint64_t o = ((uint64_t)s * a.P + p) * a.k + (h - s * a.k);
        if (a.dgamma) a.dgamma[o] = g[i];
        if (a.dbeta) a.dbeta[o] = b[i];
    }
}

static bool on(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Bytes of the widest load that all rows begin on and that divides a row: 16, or 4 or 2 (the element) where that does not fit.
static uint32_t row_vector(const NormArgs& a) {
    const uint32_t e = a.dtype == FTC_F32 ? 4 : 2;
    const uint64_t strides = (a.x_stride | a.y_stride | a.dy_stride | a.dx_stride | a.H) * e;
    const auto fits = [&](uint32_t v) { return strides % v == 0 && on(a.x, v) && on(a.y, v) && on(a.dy, v) && on(a.dx, v); };
    if (fits(16) && on(a.gamma, 16) && on(a.beta, 16)) return 16;
    return fits(4) ? 4 : e;
}

template <typename T, typename W> static cudaError_t forward(const NormArgs& a, int sms, cudaStream_t st) {
    const cudaError_t e = forward_rows<T, W>(a, row_vector(a), sms, st);
    if (e != cudaErrorNotSupported) return e;
    if (a.H <= kLongest) {
        const uint32_t threads = (a.H + 1023) / 1024 * 32, cap = (uint32_t)sms * (1024 / threads), grid = a.rows < cap ? a.rows : cap;
        if (row_vector(a) == 16) norm_forward_wide_kernel<T, W, 16><<<grid, threads, 0, st>>>(a);
        else norm_forward_wide_kernel<T, W, sizeof(T)><<<grid, threads, 0, st>>>(a);
        return cudaGetLastError();
    }
    const uint64_t cap = (uint64_t)sms * 8;
    norm_forward_long_kernel<T, W><<<(uint32_t)(a.rows < cap ? a.rows : cap), kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_norm_forward(const NormArgs& a, int sms, cudaStream_t st) {
    if (a.dtype == FTC_F32) return forward<float, float>(a, sms, st);
    if (a.dtype == FTC_BF16) return a.wdtype == FTC_F32 ? forward<__nv_bfloat16, float>(a, sms, st) : forward<__nv_bfloat16, __nv_bfloat16>(a, sms, st);
    return a.wdtype == FTC_F32 ? forward<__half, float>(a, sms, st) : forward<__half, __half>(a, sms, st);
}

// One group for each process, which writes its messages itself (no partial sums, no second kernel): for even shares on rows that fit a
// group, where a process has few rows (bf16, H = 2048, 64 processes of 4 rows: 9.6 us a call against 12.0), or not many and the processes
// alone come near what the GPU runs at once (H = 1024, 1024 processes of 16 rows: 21 us against 29). With long walks the last
// round of groups would leave the GPU half empty (H = 4096, 300 processes of 64 rows: 118 us against 87). Around the borders, us on the GPU, bf16, this
// against slots: H = 1024, 64 processes of 4, 8, 12, 16, 24 rows: 4.1, 6.1, 7.9, 9.7, 13.5 against 5.1, 6.4, 9.6, 10.1, 10.3 (a call's two launches add
// two to five more); H = 4096: 5.8, 8.3, 11.0, 13.5 against 8.4, 9.1, 10.0, 11.0; 256 processes: 7.9, 11.6, 15.4, 21.0, 29.6 against 16.6, 20.4, 24.5, 29.8, 39.1.
uint32_t norm_backward_direct(const NormArgs& a, int sms) {
    if (a.splits || !(a.dgamma || a.dbeta) || !a.rows || a.H > 16 * kMaxGroup) return 0;
    const uint32_t g = group_threads(a.H), per_sm = g < 512 ? 512 / g : 1;
    if (a.rows > 8ull * a.P && (a.rows > 16ull * a.P || 4ull * a.P < (uint64_t)sms * per_sm)) return 0;
    return a.k % 4 == 0 && on(a.dgamma, 16) && on(a.dbeta, 16) ? 2 : 1;
}

// Groups that share the rows in the backward pass: as many as the GPU runs at once. Each group writes and the second kernel reads 8 bytes a
// column: where that comes to more than 8 MB in all, groups have at least 16 rows (which keeps it under a sixth of the rows' own 96 bytes
// and more), and never partial sums of more than 2 GiB.
uint32_t norm_backward_groups(uint32_t H, uint64_t rows, int sms) {
    const uint32_t g = group_threads(H), per_sm = g < 512 ? 512 / g : 1;
    uint64_t n = (uint64_t)sms * per_sm;
    const uint64_t cheap = (1u << 20) / H, few = rows / 16 > (uint64_t)sms ? rows / 16 : (uint64_t)sms, room = (1ull << 28) / H;
    if (n > few && n > cheap) n = few > cheap ? few : cheap;
    if (n > room) n = room ? room : 1;
    if (n > rows) n = rows;
    if (n == 0) return 0;
    const uint64_t each = (rows + n - 1) / n;
    return (uint32_t)((rows + each - 1) / each);
}

template <typename T> static cudaError_t columns(const NormArgs& a, cudaStream_t st) {
    constexpr int e = sizeof(T);
    const uint32_t v = row_vector(a), threads = (a.H * e / v + kThreads - 1) / kThreads;
    const dim3 grid(threads, a.groups);
    if (v == 16) norm_columns_kernel<T, 16><<<grid, kThreads, 0, st>>>(a);
    else if (v == 4) norm_columns_kernel<T, 4><<<grid, kThreads, 0, st>>>(a);
    else norm_columns_kernel<T, e><<<grid, kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T, typename W> static cudaError_t backward(const NormArgs& a, int sms, cudaStream_t st) {
    const cudaError_t e = backward_rows<T, W>(a, row_vector(a), st);
    if (e != cudaErrorNotSupported) return e;
    if (a.slots) { const cudaError_t c = columns<T>(a, st); if (c != cudaSuccess || !a.dx) return c; }
    const uint32_t v = row_vector(a), vecs = a.H * (uint32_t)sizeof(T) / 16;
    if (v == 16 && vecs <= 4 * 1024) {
        const uint32_t threads = (vecs + 127) / 128 * 32, cap = (uint32_t)sms * (1024 / threads);
        norm_backward_long_kernel<T, W, 16, true><<<a.rows < cap ? a.rows : cap, threads, 0, st>>>(a);
    } else {
        const uint32_t cap = (uint32_t)sms * 4, grid = a.rows < cap ? a.rows : cap;
        if (v == 16) norm_backward_long_kernel<T, W, 16, false><<<grid, 512, 0, st>>>(a);
        else norm_backward_long_kernel<T, W, sizeof(T), false><<<grid, 512, 0, st>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t launch_norm_backward(const NormArgs& a, int sms, cudaStream_t st) {
    if (a.rows) {
        cudaError_t e;
        if (a.dtype == FTC_F32) e = backward<float, float>(a, sms, st);
        else if (a.dtype == FTC_BF16) e = a.wdtype == FTC_F32 ? backward<__nv_bfloat16, float>(a, sms, st) : backward<__nv_bfloat16, __nv_bfloat16>(a, sms, st);
        else e = a.wdtype == FTC_F32 ? backward<__half, float>(a, sms, st) : backward<__half, __half>(a, sms, st);
        if (e != cudaSuccess) return e;
    }
    if (!a.slots) return cudaSuccess;
    const uint32_t S = (a.H + a.k - 1) / a.k;
    const uint64_t filled = (uint64_t)S * a.k;                       // columns with the last message's fill
    const uint32_t tiles = (uint32_t)((filled + 31) / 32), wide = (uint32_t)((filled + 127) / 128), slots = a.groups / a.P + 1;    // slots of a process, on average
    const uint64_t items = (uint64_t)tiles * a.P;
    if (items > 0x7FFFFFFFull) return cudaErrorInvalidValue;         // refused before (ftc_train_api.cu)
    const uint32_t n = (uint32_t)items, nw = wide * a.P;
    if (!a.rows) {                                                   // zeros; no earlier kernel of this call
        norm_messages_kernel<1, 4><<<(nw + 7) / 8, 256, 0, st>>>(a, wide, nw);
        return cudaGetLastError();
    }
    // A warp for each process and tile where slots are few or warps plenty; four columns a lane where that still leaves every SM its 64
    // warps (955 processes of 13256 columns, two slots each: 46 us against 96).
    if (slots <= 2 && nw >= 64u * sms) return launch_second(norm_messages_kernel<1, 4>, (nw + 7) / 8, 256, st, a, wide, nw);
    if (slots <= 2 || (slots <= 12 && n >= 32u * sms)) return launch_second(norm_messages_kernel<1, 1>, (n + 7) / 8, 256, st, a, tiles, n);
    if (slots <= 12) return launch_second(norm_messages_kernel<4, 1>, (n + 1) / 2, 256, st, a, tiles, n);
    if (slots <= 64) return launch_second(norm_messages_kernel<8, 1>, n, 256, st, a, tiles, n);
    return launch_second(norm_messages_kernel<32, 1>, n, 1024, st, a, tiles, n);
}

}  // namespace ftc
