// Embedding lookup and its gradient by sorted tokens.
//
// Forward: y[t] = scale * table[token t]. A warp takes a piece of a row, 8 elements a lane; bound by memory (65536 tokens of 4096, float32 to
// bf16: 163 us, 0.93 GB through memory, what several tokens name once).
//
// Backward: the gradient of a table of V rows is dense (it is what the allreduce's messages hold), almost all of it zeros, so its bytes
// are mostly those of writing zeros. The kernels:
//   1. one cluster sorts the tokens (a stable radix sort by value, 8 bits a pass, so that equal tokens keep their order, and with it
//      the order of processes); the rest of the GPU writes zeros to the whole gradient meanwhile, a kernel of its own;
//   2. the sorted list is cut into chunks of 32; a warp sums a chunk's rows of dy for its 256 columns, run by run (a run: one token of one
//      process), and writes the runs that lie inside the chunk where they belong, sums of the others to the workspace;
//   3. runs that cross chunks: the first chunk's sum and the following ones' in order, shared out over the warps of a block.
// 32768 tokens of 1024 in bf16 for 8 processes of 32768 x 1024: 185 us, of which 146 zeros (the sorting's 26 beside them), 29 and 9.
// Whatever the tokens' distribution, all warps of step 2 have 32 rows to sum. No atomic addition takes part. Few tokens are not sorted.
#include <cooperative_groups.h>
#include "ftc_lm.cuh"

namespace ftc {

constexpr uint32_t kChunk = FTC_EMBED_RUN;                       // entries of the sorted list that a warp sums
constexpr uint32_t kPiece = 256;                                 // columns of a warp
constexpr uint32_t kSortThreads = 1024, kSortWarps = kSortThreads / 32, kItems = 4, kTile = kSortThreads * kItems;
constexpr uint32_t kCuts = 1024;                                 // splits that are kept in shared memory
constexpr uint32_t kHeldBytes = kTile * 8;

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

// Zeros, 32 KB a block in stores of 32 bytes: many short blocks, one after the other through memory (7.3 TB/s; blocks that stride through all of
// it made 5.5, copies out of zeroed shared memory 4.2). The sorting goes on meanwhile: one thread waits for it.
constexpr uint32_t kZeroThreads = 256, kZeroFloats = 8192;
__global__ void __launch_bounds__(kZeroThreads) zero_kernel(float* out, uint64_t n, uint32_t sorting) {
    later_kernel_may_start();
    const uint64_t ahead = min(n, (uint64_t)((32 - (reinterpret_cast<uintptr_t>(out) & 31)) & 31) / 4), eights = (n - ahead) / 8, behind = ahead + eights * 8;
    float* const p = out + ahead;
    const uint64_t i0 = (uint64_t)blockIdx.x * (kZeroFloats / 8) + threadIdx.x;
#pragma unroll
    for (uint32_t j = 0; j < kZeroFloats / 8 / kZeroThreads; ++j) {
        const uint64_t i = i0 + j * kZeroThreads;
        if (i < eights) asm volatile("st.global.v8.b32 [%0], {%1,%1,%1,%1,%1,%1,%1,%1};" ::"l"(p + i * 8), "r"(0) : "memory");
    }
    if (blockIdx.x == 0) {
        if (threadIdx.x < ahead) out[threadIdx.x] = 0.f;
        if (behind + threadIdx.x < n) out[behind + threadIdx.x] = 0.f;
        if (sorting) wait_for_earlier_kernel();
    }
}

// The process that holds token t: the one whose rows splits[p] .. splits[p+1]-1 (or even shares) it is among; -1: none.
template <typename S> __device__ __forceinline__ int32_t process_among(const S* splits, uint32_t P, uint32_t t) {
    if (t < splits[0] || t >= splits[P]) return -1;
    uint32_t lo = 0, hi = P;                                     // splits[lo] <= t < splits[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (splits[mid] <= t) lo = mid; else hi = mid;
    }
    return (int32_t)lo;
}
__device__ __forceinline__ int32_t process_of(const EmbedArgs& a, uint32_t t) {
    if (!a.splits) return a.P == 1 ? 0 : (int32_t)((((uint64_t)t + 1) * a.P - 1) / a.n);
    return process_among(a.splits, a.P, t);
}

// One cluster sorts (token, position) by token in `passes` passes of 8 bits; tokens that count for nobody have the value V and come last.
//
// A block of the cluster has one stretch of the list, in each pass. It counts its digits, reads all blocks' counts, and gives every entry
// its place: entries with smaller digits, then those of earlier blocks, of earlier tiles, of earlier warps, of earlier rounds and lanes.
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(EmbedArgs a, uint32_t passes) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t C = cluster.num_blocks(), rank = cluster.block_rank(), tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    later_kernel_may_start();
    extern __shared__ __align__(16) unsigned char held_raw[];
    __shared__ uint32_t counts[2][256], base[256], sums[8];
    __shared__ __align__(128) uint32_t per_warp[kSortWarps][256];
    const uint32_t each = ((a.n + C - 1) / C + 31) & ~31u;       // n is at most 2^31: no sum here passes 32 bits
    const uint32_t begin = min(a.n, rank * each), end = min(a.n, begin + each);
    __shared__ uint32_t cuts[kCuts + 1];
    const bool near = a.splits && a.P <= kCuts;
    if (near) for (uint32_t p = tid; p <= a.P; p += kSortThreads) cuts[p] = (uint32_t)min((uint64_t)a.n, a.splits[p]);
    __syncthreads();
    auto process_at = [&](uint32_t i) { return (uint32_t)(near ? process_among(cuts, a.P, i) : process_of(a, i)); };
    auto token_key = [&](uint32_t i) -> uint32_t {
        int32_t t = token_at(a.tokens, a.token_bits, i, a.V);
        if (a.splits && (near ? i < cuts[0] || i >= cuts[a.P] : i < a.splits[0] || i >= a.splits[a.P])) t = -1;
        return t < 0 ? a.V : (uint32_t)t;
    };
    // Places of the smaller digits and of the earlier blocks' same ones, from all blocks' counts.
    auto places = [&](const uint32_t* count) {
        if (tid < 256) {
            uint32_t total = 0, before = 0;
            for (uint32_t b = 0; b < C; ++b) {
                const uint32_t c = cluster.map_shared_rank(const_cast<uint32_t*>(count), b)[tid];
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
    };
    if (each <= kTile) {
        // A block's entries stay in registers and, between passes, in the blocks' shared memory.
        uint32_t* const held = reinterpret_cast<uint32_t*>(held_raw);            // keys, then positions
        uint32_t key[kItems], index[kItems], place[kItems];
#pragma unroll
        for (uint32_t j = 0; j < kItems; ++j) {
            index[j] = begin + warp * (32 * kItems) + j * 32 + lane;
            key[j] = index[j] < end ? token_key(index[j]) : 0xFFFFFFFFu;
        }
        for (uint32_t pass = 0; pass < passes; ++pass) {
            const uint32_t shift = pass * 8;
            uint32_t* const count = counts[pass & 1];
            auto there = [&](uint32_t j) { return begin + warp * (32 * kItems) + j * 32 + lane < end; };
            for (uint32_t d = lane; d < 256; d += 32) per_warp[warp][d] = 0;
            __syncwarp();
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                const uint32_t digit = there(j) ? key[j] >> shift & 255u : 256u;
                const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit), before = __popc(same & ((1u << lane) - 1));
                place[j] = digit < 256 ? per_warp[warp][digit] + before : 0;
                __syncwarp();
                if (digit < 256 && before == 0) per_warp[warp][digit] += __popc(same);
                __syncwarp();
            }
            __syncthreads();
            {                                                    // four threads a digit, eight warps each
                const uint32_t d = tid / 4, w0 = tid % 4 * 8;
                uint32_t c[8], all = 0;
#pragma unroll
                for (uint32_t w = 0; w < 8; ++w) { c[w] = per_warp[w0 + w][d]; all += c[w]; }
                uint32_t run = all;
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, run, o, 4);
                    if (tid % 4 >= (uint32_t)o) run += up;
                }
                if (tid % 4 == 3) count[d] = run;
                run -= all;
#pragma unroll
                for (uint32_t w = 0; w < 8; ++w) { per_warp[w0 + w][d] = run; run += c[w]; }
            }
            cluster.sync();
            places(count);
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                if (!there(j)) continue;
                const uint32_t d = key[j] >> shift & 255u, to = base[d] + per_warp[warp][d] + place[j];
                if (pass + 1 == passes) {
                    a.keys[0][to] = key[j]; a.index[0][to] = index[j]; a.process[to] = process_at(index[j]);
                } else {
                    const uint32_t b = to / each;
                    uint32_t* const h = cluster.map_shared_rank(held, b);
                    h[to - b * each] = key[j]; h[kTile + to - b * each] = index[j];
                }
            }
            if (pass + 1 == passes) break;
            cluster.sync();
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j)
                if (there(j)) { const uint32_t i = warp * (32 * kItems) + j * 32 + lane; key[j] = held[i]; index[j] = held[kTile + i]; }
        }
        cluster.sync();                                          // a block's shared memory stays until all have read it
        return;
    }
    for (uint32_t pass = 0; pass < passes; ++pass) {
        const uint32_t shift = pass * 8, side = (passes - 1 - pass) & 1;
        uint32_t* const count = counts[pass & 1];
        const uint32_t* const from_key = a.keys[side ^ 1];
        const uint32_t* const from_index = a.index[side ^ 1];
        auto key_at = [&](uint32_t i) -> uint32_t { return pass ? __ldcg(from_key + i) : token_key(i); };
        if (tid < 256) count[tid] = 0;
        __syncthreads();
        for (uint32_t i0 = begin + warp * 32; i0 < end; i0 += kSortThreads) {
            const uint32_t i = i0 + lane, digit = i < end ? key_at(i) >> shift & 255u : 256u;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
            if (digit < 256 && lane == (uint32_t)__ffs(same) - 1) atomicAdd(&count[digit], __popc(same));
        }
        cluster.sync();
        places(count);
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
                    if (pass + 1 == passes) a.process[to] = process_at(index);
                }
            }
            __syncthreads();
        }
        cluster.sync();
    }
}

// ---- backward: sums of runs ----

// A lane's columns of a warp's piece: eight neighbours (WIDE, pieces of 256) or two that lie 32 apart (pieces of 64: rows on any address, and
// more warps for the short rows that odd widths are). Rows are loaded as they are, several ahead, and become numbers when they are added.
template <typename T, bool WIDE> struct Columns;
template <typename T> struct Columns<T, true> {
    static constexpr uint32_t kCols = 8, kPieceCols = 256, kAhead = sizeof(T) == 2 ? 8 : 4;
    struct Raw { uint4 r[sizeof(T) / 2]; };
    static __device__ __forceinline__ bool has(uint32_t lane, uint32_t left) { return lane * 8 < left; }
    static __device__ __forceinline__ void load(Raw& w, const T* row, uint32_t lane, uint32_t left) {
        if (!has(lane, left)) return;
        const uint4* p = reinterpret_cast<const uint4*>(row + lane * 8);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w.r[i] = __ldg(p + i);
    }
    static __device__ __forceinline__ void add(float* v, const Raw& w, bool fresh) {
        float x[8];
        load8(x, reinterpret_cast<const T*>(w.r));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fresh ? x[i] : v[i] + x[i];
    }
    static __device__ __forceinline__ void add_floats(float* v, const float* row, uint32_t lane, uint32_t left) {
        if (!has(lane, left)) return;
        float x[8];
        load8(x, row + lane * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += x[i];
    }
    static __device__ __forceinline__ void store(float* row, const float* v, uint32_t lane, uint32_t left) {
        if (has(lane, left)) store8(row + lane * 8, v);
    }
};
template <typename T> struct Columns<T, false> {
    static constexpr uint32_t kCols = 2, kPieceCols = 64, kAhead = 16;
    struct Raw { T r[2]; };
    static __device__ __forceinline__ void load(Raw& w, const T* row, uint32_t lane, uint32_t left) {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
            if (lane + i * 32 < left) w.r[i] = row[lane + i * 32];
    }
    static __device__ __forceinline__ void add(float* v, const Raw& w, bool fresh) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = fresh ? to_f32(w.r[i]) : v[i] + to_f32(w.r[i]);
    }
    static __device__ __forceinline__ void add_floats(float* v, const float* row, uint32_t lane, uint32_t left) {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
            if (lane + i * 32 < left) v[i] += row[lane + i * 32];
    }
    static __device__ __forceinline__ void store(float* row, const float* v, uint32_t lane, uint32_t left) {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
            if (lane + i * 32 < left) row[lane + i * 32] = v[i];
    }
};

// The message of place r (counted from the beginning of a message that a piece begins in): r / k. Pieces are shorter than 4096, and r is below
// k + 4096: with a k of that at most, r * k stays below 2^32, which makes the multiplication exact.
__device__ __forceinline__ uint32_t messages_on(const EmbedArgs& a, uint32_t r) { return a.k < 4096 ? __umulhi(r, a.k_inverse) + (a.k == 1 ? r : 0) : r >= a.k; }

// The gradient's row v of process p, columns from c on: where the messages have them.
template <typename T, bool WIDE> __device__ __forceinline__ void store_messages(const EmbedArgs& a, uint32_t v, uint32_t p, uint32_t c, float* x, uint32_t lane, uint32_t left) {
    using Cols = Columns<T, WIDE>;
    const uint64_t e = (uint64_t)v * a.H + c;
#pragma unroll
    for (uint32_t j = 0; j < Cols::kCols; ++j) x[j] *= a.scale;
    if (a.P == 1) { Cols::store(a.dtable + e, x, lane, left); return; }
    const uint64_t s0 = a.k_shift < 32 ? e >> a.k_shift : e / a.k;
    const uint32_t r0 = (uint32_t)(e - s0 * a.k);
    float* const out = a.dtable + (s0 * a.P + p) * a.k;
    if (WIDE) {                                                  // k, H and the address allow vectors of four (launch_embedding_backward)
        if (lane * 8 >= left) return;
#pragma unroll
        for (uint32_t q = 0; q < 2; ++q) {
            const uint32_t r = r0 + lane * 8 + q * 4, s = messages_on(a, r);
            *reinterpret_cast<float4*>(out + (uint64_t)s * a.P * a.k + (r - s * a.k)) = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < Cols::kCols; ++j)
            if (lane + j * 32 < left) {
                const uint32_t r = r0 + lane + j * 32, s = messages_on(a, r);
                out[(uint64_t)s * a.P * a.k + (r - s * a.k)] = x[j];
            }
    }
}

template <typename T, bool WIDE> __global__ void __launch_bounds__(128) sum_runs_kernel(EmbedArgs a, uint32_t pieces, uint32_t units) {
    using Cols = Columns<T, WIDE>;
    wait_for_earlier_kernel();
    later_kernel_may_start();
    const uint32_t lane = threadIdx.x % 32, u = blockIdx.x * 4 + threadIdx.x / 32;
    if (u >= units) return;
    const uint32_t chunk = u / pieces, c = (u - chunk * pieces) * Cols::kPieceCols, left = a.H - c;
    const uint32_t b = chunk * kChunk, i = b + lane, m = min(kChunk, a.n - b);
    const bool there = lane < m;
    const uint32_t key = there ? a.keys[0][i] : a.V, index = there ? a.index[0][i] : 0, process = there ? a.process[i] : 0;
    // does the entry continue the run of the one before it; does the entry behind the chunk continue the last one's
    const uint32_t key_before = i && there ? a.keys[0][i - 1] : 0xFFFFFFFFu, process_before = i && there ? a.process[i - 1] : 0;
    const uint32_t key_behind = b + m < a.n ? a.keys[0][b + m] : 0xFFFFFFFFu, process_behind = b + m < a.n ? a.process[b + m] : 0;
    const uint32_t goes_on = __ballot_sync(0xFFFFFFFFu, there && key == key_before && process == process_before);
    const uint32_t live = __popc(__ballot_sync(0xFFFFFFFFu, key < a.V));         // those that count for nobody come last
    const uint32_t last = m - 1, key_last = __shfl_sync(0xFFFFFFFFu, key, last), process_last = __shfl_sync(0xFFFFFFFFu, process, last);
    const bool leaves = key_behind == key_last && process_behind == process_last;
    const T* const dy = static_cast<const T*>(a.dy) + c;
    float sum[Cols::kCols];
    for (uint32_t e0 = 0; e0 < live; e0 += Cols::kAhead) {
        typename Cols::Raw raw[Cols::kAhead];
#pragma unroll
        for (uint32_t j = 0; j < Cols::kAhead; ++j) {
            const uint32_t row = __shfl_sync(0xFFFFFFFFu, index, (e0 + j) & 31);
            if (e0 + j < live) Cols::load(raw[j], dy + (uint64_t)row * a.dy_stride, lane, left);
        }
#pragma unroll
        for (uint32_t j = 0; j < Cols::kAhead; ++j) {
            const uint32_t e = e0 + j;
            if (e >= live) break;
            Cols::add(sum, raw[j], e == 0 || !(goes_on >> e & 1u));
            if (e != last && (goes_on >> (e + 1) & 1u)) continue;
            const uint32_t k = __shfl_sync(0xFFFFFFFFu, key, e), p = __shfl_sync(0xFFFFFFFFu, process, e);
            const uint32_t all = (2u << e) - 1;                  // the run began before this chunk if all its entries up to the first go on
            if ((goes_on & all) == all) Cols::store(a.parts + (uint64_t)chunk * 2 * a.H + c, sum, lane, left);
            else if (e == last && leaves) Cols::store(a.parts + ((uint64_t)chunk * 2 + 1) * a.H + c, sum, lane, left);
            else store_messages<T, WIDE>(a, k, p, c, sum, lane, left);
        }
    }
}

// Runs that begin in one chunk and end in a later one: a block for each chunk's last run. A warp takes a piece of the columns; where a run is
// long, the block's warps share its chunks, and the sums of the eight parts are added in order.
template <bool WIDE> __global__ void __launch_bounds__(256) join_runs_kernel(EmbedArgs a, uint32_t pieces) {
    using Cols = Columns<float, WIDE>;
    constexpr uint32_t kLong = 16;                               // chunks
    wait_for_earlier_kernel();
    const uint32_t chunk = blockIdx.x, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t next = (chunk + 1) * kChunk;
    const uint32_t key = a.keys[0][next], process = a.process[next], key_here = a.keys[0][next - 1], process_here = a.process[next - 1];
    const uint32_t key_first = chunk ? a.keys[0][next - kChunk - 1] : 0xFFFFFFFFu, process_first = chunk ? a.process[next - kChunk - 1] : 0;
    if (key >= a.V || key_here != key || process_here != process) return;        // nothing leaves this chunk
    if (key_first == key && process_first == process) return;                    // began further before
    // the run's last chunk: the first one behind whose end another run begins
    __shared__ uint32_t found;
    __shared__ float sums[8][Cols::kCols][32];
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
    const uint32_t n = to - chunk;
    const float* const parts = a.parts;
    const uint64_t step = 2 * (uint64_t)a.H;
    if (n <= kLong) {
        for (uint32_t piece = warp; piece < pieces; piece += 8) {
            const uint32_t c = piece * Cols::kPieceCols, left = a.H - c;
            float sum[Cols::kCols] = {};
            Cols::add_floats(sum, parts + (uint64_t)chunk * step + a.H + c, lane, left);
#pragma unroll 8
            for (uint32_t q = 1; q <= n; ++q) Cols::add_floats(sum, parts + (chunk + q) * step + c, lane, left);
            store_messages<float, WIDE>(a, key, process, c, sum, lane, left);
        }
        return;
    }
    const uint32_t each = (n + 7) / 8, q0 = 1 + warp * each, q1 = min(n + 1, q0 + each);
    for (uint32_t piece = 0; piece < pieces; ++piece) {
        const uint32_t c = piece * Cols::kPieceCols, left = a.H - c;
        float sum[Cols::kCols] = {};
        if (warp == 0) Cols::add_floats(sum, parts + (uint64_t)chunk * step + a.H + c, lane, left);
#pragma unroll 8
        for (uint32_t q = q0; q < q1; ++q) Cols::add_floats(sum, parts + (chunk + q) * step + c, lane, left);
#pragma unroll
        for (uint32_t j = 0; j < Cols::kCols; ++j) sums[warp][j][lane] = sum[j];
        __syncthreads();
        if (warp == piece % 8) {                                 // another warp each time
#pragma unroll
            for (uint32_t j = 0; j < Cols::kCols; ++j) {
                sum[j] = sums[0][j][lane];
                for (uint32_t w = 1; w < 8; ++w) sum[j] += sums[w][j][lane];
            }
            store_messages<float, WIDE>(a, key, process, c, sum, lane, left);
        }
        __syncthreads();
    }
}

// Few tokens (256 WORDS, kFew at most) need no sorting: a block for each token and piece of its columns, which goes on if the token is the first of its value
// in its process (or for some of its pieces). Its eight warps look through an eighth of the process's tokens each and sum what they find, eight
// rows ahead.
constexpr uint32_t kFew = 2048;                                  // measured up to there: 2000 tokens 27 us sorted, 19 so; 4096 33 against 67
template <typename T, bool WIDE, uint32_t WORDS> __global__ void __launch_bounds__(256) sum_few_kernel(EmbedArgs a, uint32_t pieces) {
    using Cols = Columns<T, WIDE>;
    const uint32_t t = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int32_t token = token_at(a.tokens, a.token_bits, t, a.V), p = process_of(a, t);
    // the process's tokens
    uint32_t first = 0, end = a.n;
    if (p >= 0 && a.splits) {
        first = (uint32_t)min((uint64_t)a.n, a.splits[p]); end = (uint32_t)min((uint64_t)a.n, a.splits[p + 1]);
    } else if (p >= 0 && a.P > 1) {
        first = (uint32_t)((uint64_t)p * a.n / a.P); end = (uint32_t)(((uint64_t)p + 1) * a.n / a.P);
    }
    const uint32_t each = ((end - first + 7) / 8 + 31) & ~31u, i0 = first + warp * each, i1 = min(end, i0 + each);      // i0 may lie behind the end
    uint32_t found[WORDS] = {};                             // bits of this warp's tokens that are the same
    bool earlier = false;
#pragma unroll
    for (uint32_t w = 0; w < WORDS; ++w) {
        const uint32_t i = i0 + w * 32 + lane;
        const bool same = i < i1 && token_at(a.tokens, a.token_bits, i, a.V) == token;
        found[w] = __ballot_sync(0xFFFFFFFFu, same);
        earlier |= same && i < t;
    }
    const bool none = __syncthreads_or(earlier || token < 0 || p < 0);
    wait_for_earlier_kernel();                                   // the zeros
    if (none) return;
    __shared__ float sums[8][Cols::kCols][32];
    for (uint32_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const uint32_t c = piece * Cols::kPieceCols, left = a.H - c;
        const T* const dy = static_cast<const T*>(a.dy) + c;
        float sum[Cols::kCols] = {};
#pragma unroll
        for (uint32_t w = 0; w < WORDS; ++w) {
            uint32_t bits = found[w];
            while (bits) {
                typename Cols::Raw raw[Cols::kAhead];
                uint32_t rest = bits;
#pragma unroll
                for (uint32_t j = 0; j < Cols::kAhead; ++j) {
                    if (rest) Cols::load(raw[j], dy + (uint64_t)(i0 + w * 32 + __ffs(rest) - 1) * a.dy_stride, lane, left);
                    rest &= rest - 1;
                }
#pragma unroll
                for (uint32_t j = 0; j < Cols::kAhead; ++j) {
                    if (bits) Cols::add(sum, raw[j], false);
                    bits &= bits - 1;
                }
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < Cols::kCols; ++j) sums[warp][j][lane] = sum[j];
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (uint32_t j = 0; j < Cols::kCols; ++j)
                for (uint32_t w = 1; w < 8; ++w) sum[j] += sums[w][j][lane];
            store_messages<T, WIDE>(a, (uint32_t)token, (uint32_t)p, c, sum, lane, left);
        }
        __syncthreads();
    }
}

template <typename T, bool WIDE> static cudaError_t sums(const EmbedArgs& a, bool few, int sms, cudaStream_t st) {
    const uint32_t cols = Columns<T, WIDE>::kPieceCols, pieces = (a.H + cols - 1) / cols, chunks = (a.n + kChunk - 1) / kChunk;
    if (few) {                                                   // no more blocks than the GPU has room for, once there is one for each token
        const uint32_t most = ((uint32_t)sms * 8 + a.n - 1) / a.n;
        const dim3 grid(pieces < most ? pieces : most, a.n);
        return a.n <= 1024 ? launch_second(sum_few_kernel<T, WIDE, 4>, grid, 256, st, a, pieces) : launch_second(sum_few_kernel<T, WIDE, 8>, grid, 256, st, a, pieces);
    }
    const uint64_t units = (uint64_t)chunks * pieces;
    if (units > 0x7FFFFFFFull) return cudaErrorInvalidValue;     // refused before (ftc_lm_api.cu)
    cudaError_t e = launch_second(sum_runs_kernel<T, WIDE>, (uint32_t)((units + 3) / 4), 128, st, a, pieces, (uint32_t)units);
    if (e != cudaSuccess || chunks < 2) return e;
    return launch_second(join_runs_kernel<WIDE>, chunks - 1, 256, st, a, pieces);
}

cudaError_t launch_embedding_backward(const EmbedArgs& args, int sms, cudaStream_t st) {
    EmbedArgs a = args;
    a.k_shift = a.k & (a.k - 1) ? 32 : (uint32_t)__builtin_ctz(a.k);
    a.k_inverse = (uint32_t)(((1ull << 32) + a.k - 1) / a.k);
    const bool few = a.n <= kFew;
    const uint32_t zeros = (uint32_t)((a.out_floats + kZeroFloats - 1) / kZeroFloats);
    cudaError_t e;
    if (few) {
        zero_kernel<<<zeros, kZeroThreads, 0, st>>>(a.dtable, a.out_floats, 0);
        e = cudaGetLastError();
    } else {
        // One block sorts up to a tile; a cluster of eight beyond.
        uint32_t passes = 1;
        while (passes < 4 && a.V >> (8 * passes)) ++passes;
        cudaLaunchAttribute shape{};
        shape.id = cudaLaunchAttributeClusterDimension;
        shape.val.clusterDim.x = a.n > kTile ? 8 : 1; shape.val.clusterDim.y = shape.val.clusterDim.z = 1;
        cudaLaunchConfig_t how{};
        how.gridDim = dim3(shape.val.clusterDim.x); how.blockDim = dim3(kSortThreads); how.dynamicSmemBytes = kHeldBytes; how.stream = st; how.attrs = &shape; how.numAttrs = 1;
        e = cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldBytes);
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&how, sort_tokens_kernel, a, passes);
        if (e == cudaSuccess) e = launch_second(zero_kernel, zeros, kZeroThreads, st, a.dtable, a.out_floats, 1u);
    }
    if (e != cudaSuccess || !a.n) return e;
    const uint64_t es = a.dtype == FTC_F32 ? 4 : 2;
    const bool wide = a.H % 8 == 0 && (a.k % 4 == 0 || a.P == 1) && on16(a.dy, a.dy_stride * es) && on16(a.dtable, 0);
    if (a.dtype == FTC_F32) return wide ? sums<float, true>(a, few, sms, st) : sums<float, false>(a, few, sms, st);
    if (a.dtype == FTC_BF16) return wide ? sums<__nv_bfloat16, true>(a, few, sms, st) : sums<__nv_bfloat16, false>(a, few, sms, st);
    return wide ? sums<__half, true>(a, few, sms, st) : sums<__half, false>(a, few, sms, st);
}

}  // namespace ftc
