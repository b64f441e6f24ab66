// Embedding lookup and its gradient by sorted tokens.
//
// Forward: y[t] = scale * table[token t]. A warp takes a piece of a row, 8 elements a lane; bound by memory.
//
// Backward: the gradient of a table of V rows is dense (it is what the allreduce's messages hold), almost all of it zeros, so its bytes
// are mostly those of writing zeros. Three kernels:
//   1. one cluster sorts the tokens (a stable radix sort by value, 8 bits a pass, so that equal tokens keep their order, and with it
//      the order of processes); all other blocks write zeros to the whole gradient meanwhile;
//   2. the sorted list is cut into chunks of 32; a warp sums a chunk's rows of dy for its 256 columns, run by run (a run: one token of one
//      process), and writes the runs that lie inside the chunk where they belong, sums of the others to the workspace;
//   3. runs that cross chunks: the first chunk's sum and the following ones' in order, shared out over the warps of a block.
// Whatever the tokens' distribution, all warps of step 2 have 32 rows to sum. No atomic addition takes part.
#include <cooperative_groups.h>
#include "ftc_lm.cuh"

namespace ftc {

constexpr uint32_t kChunk = FTC_EMBED_RUN;                       // entries of the sorted list that a warp sums
constexpr uint32_t kPiece = 256;                                 // columns of a warp
constexpr uint32_t kSortThreads = 1024, kSortWarps = kSortThreads / 32, kItems = 4, kTile = kSortThreads * kItems;

// ---- eight neighbouring elements ----

__device__ __forceinline__ void load8(float* v, const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void spread(float* v, uint4 r, __nv_bfloat16) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void spread(float* v, uint4 r, __half) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}
template <typename T> __device__ __forceinline__ void load8(float* v, const T* p) { spread(v, *reinterpret_cast<const uint4*>(p), T()); }
__device__ __forceinline__ void store8(float* p, const float* v) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float* v) {
    uint4 r;
    uint32_t* w = &r.x;
    T h[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[0] = from_f32<T>(v[2 * i]); h[1] = from_f32<T>(v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(h);
    }
    *reinterpret_cast<uint4*>(p) = r;
}

// ---- forward ----

// Eight elements of a lane: neighbours (WIDE) or 32 apart.
template <typename T, typename W, bool WIDE> __global__ void __launch_bounds__(256) embedding_forward_kernel(EmbedArgs a) {
    const uint32_t lane = threadIdx.x % 32, pieces = (a.H + kPiece - 1) / kPiece;
    const uint64_t units = (uint64_t)a.n * pieces, step = (uint64_t)gridDim.x * 8;
    for (uint64_t u = (uint64_t)blockIdx.x * 8 + threadIdx.x / 32; u < units; u += step) {
        const uint32_t t = (uint32_t)(u / pieces), c = (uint32_t)(u - (uint64_t)t * pieces) * kPiece;
        const int32_t tok = token_at(a.tokens, a.token_bits, t, a.V);
        const W* src = static_cast<const W*>(a.table) + (uint64_t)(tok < 0 ? 0 : tok) * a.table_stride + c;
        T* dst = static_cast<T*>(a.y) + t * a.y_stride + c;
        float v[8];
        if (WIDE) {
            if (c + lane * 8 >= a.H) continue;
            if (tok >= 0) load8(v, src + lane * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = tok >= 0 ? v[j] * a.scale : 0.f;
            store8(dst + lane * 8, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = tok >= 0 && c + lane + j * 32 < a.H ? to_f32(src[lane + j * 32]) * a.scale : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + lane + j * 32 < a.H) dst[lane + j * 32] = from_f32<T>(v[j]);
        }
    }
}

static bool on16(const void* p, uint64_t stride_bytes) { return ((reinterpret_cast<uintptr_t>(p) | stride_bytes) & 15) == 0; }

template <typename T, typename W> static cudaError_t forward(const EmbedArgs& a, int sms, cudaStream_t st) {
    const uint64_t warps = (uint64_t)a.n * ((a.H + kPiece - 1) / kPiece), blocks = (warps + 7) / 8, cap = (uint64_t)sms * 64;
    const uint32_t grid = (uint32_t)(blocks < cap ? blocks : cap);
    const bool wide = a.H % 8 == 0 && on16(a.table, a.table_stride * sizeof(W)) && on16(a.y, a.y_stride * sizeof(T));
    if (wide) embedding_forward_kernel<T, W, true><<<grid, 256, 0, st>>>(a);
    else embedding_forward_kernel<T, W, false><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_embedding_forward(const EmbedArgs& a, int sms, cudaStream_t st) {
    if (a.dtype == FTC_F32) return forward<float, float>(a, sms, st);
    if (a.dtype == FTC_BF16) return a.wdtype == FTC_F32 ? forward<__nv_bfloat16, float>(a, sms, st) : forward<__nv_bfloat16, __nv_bfloat16>(a, sms, st);
    return a.wdtype == FTC_F32 ? forward<__half, float>(a, sms, st) : forward<__half, __half>(a, sms, st);
}

// ---- backward: the tokens sorted, zeros written ----

// The process that holds token t: the one whose rows splits[p] .. splits[p+1]-1 (or even shares) it is among; -1: none.
__device__ int32_t process_of(const EmbedArgs& a, uint32_t t) {
    if (!a.splits) return a.P == 1 ? 0 : (int32_t)((((uint64_t)t + 1) * a.P - 1) / a.n);
    if (t < a.splits[0] || t >= a.splits[a.P]) return -1;
    uint32_t lo = 0, hi = a.P;                                   // splits[lo] <= t < splits[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (a.splits[mid] <= t) lo = mid; else hi = mid;
    }
    return (int32_t)lo;
}

// The first cluster sorts (token, position) by token in `passes` passes of 8 bits; tokens that count for nobody have the value V and
// come last. All blocks of the other clusters write zeros.
//
// A block of the cluster has one stretch of the list, in each pass. It counts its digits, reads all blocks' counts, and gives every entry
// its place: entries with smaller digits, then those of earlier blocks, of earlier tiles, of earlier warps, of earlier rounds and lanes.
__global__ void __launch_bounds__(kSortThreads) sort_and_zero_kernel(EmbedArgs a, uint32_t passes) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t C = cluster.num_blocks(), rank = cluster.block_rank(), tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    later_kernel_may_start();
    if (blockIdx.x >= C) {                                       // zeros, 16 bytes a thread and store
        const uint64_t quads = a.out_floats / 4, step = (uint64_t)(gridDim.x - C) * kSortThreads;
        const uint64_t i0 = (uint64_t)(blockIdx.x - C) * kSortThreads + tid;
        if ((reinterpret_cast<uintptr_t>(a.dtable) & 15) == 0) {
            float4* out = reinterpret_cast<float4*>(a.dtable);
            for (uint64_t i = i0; i < quads; i += step) out[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i0 < a.out_floats % 4) a.dtable[quads * 4 + i0] = 0.f;
        } else {
            for (uint64_t i = i0; i < a.out_floats; i += step) a.dtable[i] = 0.f;
        }
        return;
    }
    __shared__ uint32_t counts[2][256], base[256], per_warp[kSortWarps][256], sums[8];
    const uint32_t each = ((a.n + C - 1) / C + 31) & ~31u;       // n is at most 2^31: no sum here passes 32 bits
    const uint32_t begin = min(a.n, rank * each), end = min(a.n, begin + each);
    for (uint32_t pass = 0; pass < passes; ++pass) {
        const uint32_t shift = pass * 8, side = (passes - 1 - pass) & 1;
        uint32_t* const count = counts[pass & 1];
        const uint32_t* const from_key = a.keys[side ^ 1];
        const uint32_t* const from_index = a.index[side ^ 1];
        auto key_at = [&](uint32_t i) -> uint32_t {
            if (pass) return __ldcg(from_key + i);
            int32_t t = token_at(a.tokens, a.token_bits, i, a.V);
            if (a.splits && (i < a.splits[0] || i >= a.splits[a.P])) t = -1;
            return t < 0 ? a.V : (uint32_t)t;
        };
        if (tid < 256) count[tid] = 0;
        __syncthreads();
        for (uint32_t i0 = begin + warp * 32; i0 < end; i0 += kSortThreads) {
            const uint32_t i = i0 + lane, digit = i < end ? key_at(i) >> shift & 255u : 256u;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
            if (digit < 256 && lane == (uint32_t)__ffs(same) - 1) atomicAdd(&count[digit], __popc(same));
        }
        cluster.sync();
        if (tid < 256) {                                         // places of the smaller digits and of the earlier blocks' same ones
            uint32_t total = 0, before = 0;
            for (uint32_t b = 0; b < C; ++b) {
                const uint32_t c = cluster.map_shared_rank(count, b)[tid];
                if (b < rank) before += c;
                total += c;
            }
            uint32_t run = total;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, run, o);
                if (lane >= (uint32_t)o) run += up;
            }
            if (lane == 31) sums[warp] = run;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            for (uint32_t w = 0; w < warp; ++w) run += sums[w];
            base[tid] = run - total + before;
        }
        __syncthreads();
        for (uint32_t t0 = begin; t0 < end; t0 += kTile) {
            for (uint32_t d = lane; d < 256; d += 32) per_warp[warp][d] = 0;
            __syncwarp();
            uint32_t key[kItems], place[kItems];
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                const uint32_t i = t0 + warp * (32 * kItems) + j * 32 + lane;
                key[j] = i < end ? key_at(i) : 0xFFFFFFFFu;
            }
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                const uint32_t i = t0 + warp * (32 * kItems) + j * 32 + lane, digit = i < end ? key[j] >> shift & 255u : 256u;
                const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit), before = __popc(same & ((1u << lane) - 1));
                place[j] = digit < 256 ? per_warp[warp][digit] + before : 0;
                __syncwarp();
                if (digit < 256 && before == 0) per_warp[warp][digit] += __popc(same);
                __syncwarp();
            }
            __syncthreads();
            if (tid < 256) {
                uint32_t run = base[tid];
#pragma unroll
                for (uint32_t w = 0; w < kSortWarps; ++w) { const uint32_t c = per_warp[w][tid]; per_warp[w][tid] = run; run += c; }
                base[tid] = run;
            }
            __syncthreads();
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                const uint32_t i = t0 + warp * (32 * kItems) + j * 32 + lane;
                if (i < end) {
                    const uint32_t to = per_warp[warp][key[j] >> shift & 255u] + place[j], index = pass ? __ldcg(from_index + i) : i;
                    a.keys[side][to] = key[j];
                    a.index[side][to] = index;
                    if (pass + 1 == passes) a.process[to] = (uint32_t)process_of(a, index);
                }
            }
            __syncthreads();
        }
        cluster.sync();
    }
}

// ---- backward: sums of runs ----

// Eight columns of a lane, as in the forward pass; those beyond H are not touched.
template <typename T, bool WIDE> __device__ __forceinline__ void load_columns(float* v, const T* row, uint32_t lane, uint32_t left) {
    if (WIDE) {
        if (lane * 8 < left) load8(v, row + lane * 8);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = lane + j * 32 < left ? to_f32(row[lane + j * 32]) : 0.f;
    }
}
template <bool WIDE> __device__ __forceinline__ void store_columns(float* row, const float* v, uint32_t lane, uint32_t left) {
    if (WIDE) {
        if (lane * 8 < left) store8(row + lane * 8, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (lane + j * 32 < left) row[lane + j * 32] = v[j];
    }
}

// The gradient's row v of process p, columns c .. c+255: where the messages have them.
template <bool WIDE> __device__ __forceinline__ void store_messages(const EmbedArgs& a, uint32_t v, uint32_t p, uint32_t c, const float* x, uint32_t lane, uint32_t left) {
    const uint64_t e = (uint64_t)v * a.H + c;
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j] * a.scale;
    if (a.P == 1) { store_columns<WIDE>(a.dtable + e, y, lane, left); return; }
    const uint64_t s0 = e / a.k;
    const uint32_t r0 = (uint32_t)(e - s0 * a.k);                // k and 256 together: no sum passes 32 bits
    if (WIDE) {                                                  // k, H and the address allow vectors of four (launch_embedding_backward)
        if (lane * 8 >= left) return;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t r = r0 + lane * 8 + q * 4, s = r / a.k;
            *reinterpret_cast<float4*>(a.dtable + ((s0 + s) * a.P + p) * a.k + (r - s * a.k)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (lane + j * 32 < left) {
                const uint32_t r = r0 + lane + j * 32, s = r / a.k;
                a.dtable[((s0 + s) * a.P + p) * a.k + (r - s * a.k)] = y[j];
            }
    }
}

template <typename T, bool WIDE> __global__ void __launch_bounds__(128) sum_runs_kernel(EmbedArgs a, uint32_t pieces, uint64_t units) {
    wait_for_earlier_kernel();
    later_kernel_may_start();
    const uint32_t lane = threadIdx.x % 32;
    const uint64_t u = (uint64_t)blockIdx.x * 4 + threadIdx.x / 32;
    if (u >= units) return;
    const uint32_t chunk = (uint32_t)(u / pieces), c = (uint32_t)(u - (uint64_t)chunk * pieces) * kPiece, left = a.H - c;
    const uint32_t b = chunk * kChunk, i = b + lane, m = min(kChunk, a.n - b);
    const bool there = lane < m;
    const uint32_t key = there ? a.keys[0][i] : a.V, index = there ? a.index[0][i] : 0, process = there ? a.process[i] : 0;
    // does the entry continue the run of the one before it; does the entry behind the chunk continue the last one's
    const uint32_t key_before = i && there ? a.keys[0][i - 1] : 0xFFFFFFFFu, process_before = i && there ? a.process[i - 1] : 0;
    const uint32_t goes_on = __ballot_sync(0xFFFFFFFFu, there && key == key_before && process == process_before);
    const uint32_t last = m - 1, key_last = __shfl_sync(0xFFFFFFFFu, key, last), process_last = __shfl_sync(0xFFFFFFFFu, process, last);
    const bool leaves = b + m < a.n && a.keys[0][b + m] == key_last && a.process[b + m] == process_last;
    const T* dy = static_cast<const T*>(a.dy) + c;
    float sum[8];
    constexpr uint32_t kAhead = 8;
    for (uint32_t e0 = 0; e0 < m; e0 += kAhead) {
        float v[kAhead][8];
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) {
            const uint32_t e = e0 + j, k = __shfl_sync(0xFFFFFFFFu, key, e & 31), row = __shfl_sync(0xFFFFFFFFu, index, e & 31);
            if (e < m && k < a.V) load_columns<T, WIDE>(v[j], dy + (uint64_t)row * a.dy_stride, lane, left);
        }
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) {
            const uint32_t e = e0 + j, k = __shfl_sync(0xFFFFFFFFu, key, e & 31), p = __shfl_sync(0xFFFFFFFFu, process, e & 31);
            if (e >= m || k >= a.V) continue;
            const bool fresh = e == 0 || !(goes_on >> e & 1u);
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[q] = fresh ? v[j][q] : sum[q] + v[j][q];
            const bool ends = e == last ? true : !(goes_on >> (e + 1) & 1u);
            if (!ends) continue;
            const uint32_t here = goes_on & ((2u << e) - 1);     // the run began before this chunk if all its entries up to the first go on
            const bool from_before = here == (2u << e) - 1, to_next = e == last && leaves;
            if (from_before) store_columns<WIDE>(a.parts + (uint64_t)chunk * 2 * a.H + c, sum, lane, left);
            else if (to_next) store_columns<WIDE>(a.parts + ((uint64_t)chunk * 2 + 1) * a.H + c, sum, lane, left);
            else store_messages<WIDE>(a, k, p, c, sum, lane, left);
        }
    }
}

// Runs that begin in one chunk and end in a later one: a block for each chunk's last run and 256 columns.
template <bool WIDE> __global__ void __launch_bounds__(256) join_runs_kernel(EmbedArgs a, uint32_t pieces) {
    wait_for_earlier_kernel();
    const uint32_t chunk = (uint32_t)(blockIdx.x / pieces), c = (blockIdx.x - chunk * pieces) * kPiece, left = a.H - c;
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t next = (chunk + 1) * kChunk, key = a.keys[0][next], process = a.process[next];
    if (key >= a.V || a.keys[0][next - 1] != key || a.process[next - 1] != process) return;          // nothing leaves this chunk
    if (chunk && a.keys[0][next - kChunk - 1] == key && a.process[next - kChunk - 1] == process) return;   // began further before
    // the run's last chunk: the first one behind whose end another run begins
    __shared__ uint32_t found;
    __shared__ float sums[8][kPiece];
    const uint32_t chunks = (a.n + kChunk - 1) / kChunk;
    uint32_t to = chunk + 1;
    for (;;) {                                                   // 256 chunks at a time; the list ends, and so does this
        if (threadIdx.x == 0) found = 0xFFFFFFFFu;
        __syncthreads();
        const uint32_t q = to + threadIdx.x;
        const uint64_t behind = ((uint64_t)q + 1) * kChunk;
        if (q < chunks && (behind >= a.n || a.keys[0][behind] != key || a.process[behind] != process)) atomicMin(&found, q);
        __syncthreads();
        const uint32_t f = found;
        __syncthreads();
        if (f != 0xFFFFFFFFu) { to = f; break; }
        to += 256;
    }
    // warp w has an eighth of the chunks behind the first, in order
    const uint32_t n = to - chunk, each = (n + 7) / 8, q0 = chunk + 1 + warp * each, q1 = min(to + 1, q0 + each);
    float sum[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
    if (warp == 0) load_columns<float, WIDE>(sum, a.parts + ((uint64_t)chunk * 2 + 1) * a.H + c, lane, left);
#pragma unroll 4
    for (uint32_t q = q0; q < q1; ++q) {
        load_columns<float, WIDE>(v, a.parts + (uint64_t)q * 2 * a.H + c, lane, left);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[warp][j * 32 + lane] = sum[j];
    __syncthreads();
    if (warp) return;
    for (uint32_t w = 1; w < 8 && (w * each) < n; ++w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += sums[w][j * 32 + lane];
    }
    store_messages<WIDE>(a, key, process, c, sum, lane, left);
}

template <typename T, bool WIDE> static cudaError_t sums(const EmbedArgs& a, cudaStream_t st) {
    const uint32_t pieces = (a.H + kPiece - 1) / kPiece, chunks = (a.n + kChunk - 1) / kChunk;
    const uint64_t units = (uint64_t)chunks * pieces;
    if ((units + 3) / 4 > 0x7FFFFFFFull) return cudaErrorInvalidValue;
    cudaError_t e = launch_second(sum_runs_kernel<T, WIDE>, (uint32_t)((units + 3) / 4), 128, st, a, pieces, units);
    if (e != cudaSuccess || chunks < 2) return e;
    if ((uint64_t)(chunks - 1) * pieces > 0x7FFFFFFFull) return cudaErrorInvalidValue;
    return launch_second(join_runs_kernel<WIDE>, (chunks - 1) * pieces, 256, st, a, pieces);
}

cudaError_t launch_embedding_backward(const EmbedArgs& a, int sms, cudaStream_t st) {
    // One block sorts up to a tile; a cluster of eight beyond.
    const uint32_t C = a.n > kTile ? 8 : 1;
    const uint64_t quads = (a.out_floats / 4 + kSortThreads - 1) / kSortThreads;
    uint32_t fill = (uint32_t)sms * 2;
    if (quads < fill) fill = (uint32_t)quads + 1;
    uint32_t passes = 0;                                         // no tokens: zeros only
    if (a.n) for (passes = 1; passes < 4 && a.V >> (8 * passes); ++passes) {}
    cudaLaunchAttribute shape{};
    shape.id = cudaLaunchAttributeClusterDimension;
    shape.val.clusterDim.x = C; shape.val.clusterDim.y = shape.val.clusterDim.z = 1;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3(C + (fill + C - 1) / C * C); how.blockDim = dim3(kSortThreads); how.stream = st; how.attrs = &shape; how.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&how, sort_and_zero_kernel, a, passes);
    if (e != cudaSuccess || !a.n) return e;
    const uint64_t es = a.dtype == FTC_F32 ? 4 : 2;
    const bool wide = a.H % 8 == 0 && (a.k % 4 == 0 || a.P == 1) && on16(a.dy, a.dy_stride * es) && on16(a.dtable, 0);
    if (a.dtype == FTC_F32) return wide ? sums<float, true>(a, st) : sums<float, false>(a, st);
    if (a.dtype == FTC_BF16) return wide ? sums<__nv_bfloat16, true>(a, st) : sums<__nv_bfloat16, false>(a, st);
    return wide ? sums<__half, true>(a, st) : sums<__half, false>(a, st);
}

}  // namespace ftc
