// Layer norm on rows that fit the registers of a thread block.
//
// A group of threads (a warp, or a block of up to 16 warps) holds a row, 16 elements a thread as packed pairs
// (16-bit rows of 129 to 256 on 16 bytes: one vector; other rows of up to 256 share a warp, see the narrow rows). A warp has one contiguous stretch of the row, vector i of lane l its vector 32 i + l: every load and store of a warp
// is one contiguous run, all at fixed offsets, and only the last warp may have vectors that do not exist. Statistics are taken in two
// steps from the registers (mean, then squared distances), which no common offset of the row can spoil. A group walks many rows with
// gamma, beta and the column sums in registers.
//
// Rows come in through a ring of D rows in shared memory, filled by asynchronous copies of 16 bytes that run D - 1 rows ahead: what an SM
// has under way does not depend on registers. A warp copies what it reads itself, so the ring needs no barrier of the block. Where all
// rows begin on 16 bytes (kAligned) each thread copies its own vectors. Other stretches are copied with the 16-byte pieces that cover
// them, and threads read them word by word from where they begin in the ring (kWords), 16-bit elements that begin or end between words
// as pairs out of two neighbouring words (kOdd). A piece that reaches over the array's first or last element is put together from the
// elements inside.
#pragma once
#include "ftc_f32x2.cuh"
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
    constexpr int BYTES = N * (int)sizeof(W), VB = BYTES >= 16 ? 16 : BYTES, M = VB / (int)sizeof(W);
#pragma unroll
    for (int i = 0; i < N / M; ++i) {
        Pack<W, VB> p;
        p.load(w + c + i * M);
#pragma unroll
        for (int j = 0; j < M; ++j) v[i * M + j] = p.get(j);
    }
}

// First row of process p, at most `rows`.
__device__ __forceinline__ uint32_t first_row(const NormArgs& a, uint32_t p) {
    if (!a.splits) return (uint32_t)((uint64_t)p * a.rows / a.P);
    const uint64_t s = a.splits[p];
    return s < a.rows ? (uint32_t)s : a.rows;
}

// The process that holds row r: the first one that ends behind it (P if none does); for a whole warp. Even shares: the last p with
// p*rows/P <= r. Given splits: 32 of them at a time.
__device__ __forceinline__ uint32_t holder(const NormArgs& a, uint32_t r) {
    if (!a.splits) return (uint32_t)(((uint64_t)(r + 1) * a.P - 1) / a.rows);
    uint32_t lo = 0, n = a.P;                                        // among lo .. lo + n - 1, or lo + n
    while (n) {
        const uint32_t each = (n + 31) / 32, at = (threadIdx.x & 31) * each, last = at + each < n ? at + each : n;   // a lane looks at the last of its share
        const bool behind = at < n && first_row(a, lo + last) > r;
        const uint32_t hits = __ballot_sync(0xFFFFFFFFu, behind);
        if (!hits) return lo + n;
        const uint32_t lane = __ffs(hits) - 1, from = lane * each;
        lo += from;
        n = (from + each < n ? each : n - from) - 1;                 // its last one is known to be behind
    }
    return lo;
}
// The same where process p ends before row r and a million without rows may come before the one that holds it; for a whole warp. Lane l
// looks 2^l processes ahead; what is left halves each time. (With the search above in its place the kernel for columns spilled.)
__device__ __forceinline__ uint32_t later_holder(const NormArgs& a, uint32_t p, uint32_t r) {
    if (!a.splits) return holder(a, r);
    while (true) {
        const uint32_t q = p + (1u << (threadIdx.x & 31u));           // P is at most 2^20: the last lanes are beyond it
        const uint32_t hits = __ballot_sync(0xFFFFFFFFu, q >= a.P || a.splits[q + 1] > r);
        if (hits & 1u) return p + 1;
        p += 1u << (__ffs(hits) - 2);
    }
}

// The rows of group b, and the process that holds the present one. A warp walks as one.
struct RowWalk {
    const NormArgs& a;
    uint32_t r0, r1, start, end, b, p;
    bool any;                                   // the present process has rows here so far
    __device__ __forceinline__ RowWalk(const NormArgs& args, uint32_t group) : a(args), start(0), end(~0u), b(group), p(0), any(false) {
        if (a.direct) { p = group; r0 = first_row(a, group); r1 = first_row(a, group + 1); return; }
        r0 = group * a.rows_per_group;
        r1 = a.rows - r0 < a.rows_per_group ? a.rows : r0 + a.rows_per_group;
    }
    __device__ __forceinline__ void find() { p = holder(a, r0); bounds(); }
    __device__ __forceinline__ void bounds() {
        start = p < a.P ? first_row(a, p) : ~0u;
        end = p < a.P ? first_row(a, p + 1) : ~0u;
    }
    __device__ __forceinline__ bool leaves(uint32_t r) const { return r >= end; }
    __device__ __forceinline__ void go_to(uint32_t r) {              // for the whole warp; mostly to the next process
        ++p;
        bounds();
        if (r >= end) { p = later_holder(a, p, r); bounds(); }
        any = false;
    }
    __device__ __forceinline__ bool counts(uint32_t r) const { return r >= start; }
    __device__ __forceinline__ uint64_t slot() const { return (uint64_t)b + p; }
};

// The sums of one process for N neighbouring columns, to their places in the messages.
template <int N> __device__ __forceinline__ void store_message(const NormArgs& a, uint32_t p, uint32_t c, const float* dg, const float* db) {
    if constexpr (N % 4 == 0) {
        if (a.direct == 2) {                    // messages of whole vectors of four, on 16 bytes
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                const uint32_t s = (c + j) / a.k;
                const uint64_t o = ((uint64_t)s * a.P + p) * a.k + (c + j - s * a.k);
                if (a.dgamma) *reinterpret_cast<float4*>(a.dgamma + o) = make_float4(dg[j], dg[j + 1], dg[j + 2], dg[j + 3]);
                if (a.dbeta) *reinterpret_cast<float4*>(a.dbeta + o) = make_float4(db[j], db[j + 1], db[j + 2], db[j + 3]);
            }
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (c + j >= a.H) continue;
        const uint32_t s = (c + j) / a.k;
        const uint64_t o = ((uint64_t)s * a.P + p) * a.k + (c + j - s * a.k);
        if (a.dgamma) a.dgamma[o] = dg[j];
        if (a.dbeta) a.dbeta[o] = db[j];
    }
}

template <int N> __device__ __forceinline__ void store_slot(const NormArgs& a, uint64_t slot, uint32_t c, const float* dg, const float* db) {
    float* g = a.slots + slot * 2 * a.H + c;
    float* b = g + a.H;
    if constexpr (N == 2) {                     // of an odd H every second slot begins between pairs
        if ((a.H & 1u) == 0) {
            *reinterpret_cast<float2*>(g) = make_float2(dg[0], dg[1]);
            *reinterpret_cast<float2*>(b) = make_float2(db[0], db[1]);
            return;
        }
    }
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

// Sums over the group, for all its threads. With more than one warp they go through shared memory; `turn` alternates between two places,
// so that one barrier a call is enough (a place is written again only behind the barrier of the call in between). Places of warps that
// do not exist hold zeros.
constexpr int kMaxGroup = 512, kMaxWarps = kMaxGroup / 32;
struct Scratch { float one[2][2][kMaxWarps]; };

__device__ __forceinline__ void clear_scratch(Scratch& s) {
    const uint32_t t = threadIdx.y * blockDim.x + threadIdx.x;
    if (t < 4 * kMaxWarps) (&s.one[0][0][0])[t] = 0.f;              // blocks have at least 64 threads
    __syncthreads();
}
__device__ __forceinline__ float half_warp_sum(float v) {            // of each 16 lanes
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ float group_sum(float v, Scratch& scratch, uint32_t& turn) {
    v = half_warp_sum(v);
    v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
    if (blockDim.x == 32) return v;
    float* place = scratch.one[turn][0];
    if ((threadIdx.x & 31) == 0) place[threadIdx.x >> 5] = v;
    __syncthreads();
    turn ^= 1u;
    return half_warp_sum(place[threadIdx.x & (kMaxWarps - 1)]);
}
// Two sums at once: after the first exchange the lower half of the warp goes on with x, the upper with y.
__device__ __forceinline__ float2 group_sum(float2 v, Scratch& scratch, uint32_t& turn) {
    const bool upper = threadIdx.x & 16;
    float s = (upper ? v.y : v.x) + __shfl_xor_sync(0xFFFFFFFFu, upper ? v.x : v.y, 16);
    s = half_warp_sum(s);
    if (blockDim.x != 32) {
        float(*place)[kMaxWarps] = scratch.one[turn];
        if ((threadIdx.x & 15) == 0) place[upper][threadIdx.x >> 5] = s;
        __syncthreads();
        turn ^= 1u;
        s = half_warp_sum(place[upper][threadIdx.x & (kMaxWarps - 1)]);
    }
    const float other = __shfl_xor_sync(0xFFFFFFFFu, s, 16);
    return upper ? make_float2(other, s) : make_float2(s, other);
}
__device__ __forceinline__ void group_sums(float (&v)[1], Scratch& scratch, uint32_t& turn) { v[0] = group_sum(v[0], scratch, turn); }
__device__ __forceinline__ void group_sums(float (&v)[2], Scratch& scratch, uint32_t& turn) {
    const float2 s = group_sum(make_float2(v[0], v[1]), scratch, turn);
    v[0] = s.x; v[1] = s.y;
}

// 1 / sqrt(x): the approximate one and a step of Newton's method (none at 0, infinity and NaN, where the first is right).
__device__ __forceinline__ float inverse_root(float x) {
    const float r = rsqrtf(x);
    return x > 0.f && x < 3e38f ? fmaf(r, fmaf(-0.5f * x * r, r, 0.5f), r) : r;
}

__device__ __forceinline__ void copy_async_16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_batch() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(PENDING) : "memory"); }

// A thread's part of a row: NV vectors of N elements, E in all, as pairs.
enum Mode { kAligned, kWords, kOdd };

template <typename T, int MODE, int NV_> struct Part {
    static constexpr bool SHIFT = MODE != kAligned;
    static constexpr int NV = NV_, N = SHIFT ? (sizeof(T) == 2 ? 2 : 1) : 16 / (int)sizeof(T), E = NV * N, VB = N * (int)sizeof(T);
    static_assert(E % 2 == 0, "pairs");
    static constexpr uint32_t WARP = 32 * NV, STRETCH = WARP * VB, PLACE = STRETCH + (SHIFT ? 32 : 0);   // a warp's vectors, their bytes, its room in a ring row
    static __device__ __forceinline__ uint32_t first_vector() { return (threadIdx.x >> 5) * WARP + (threadIdx.x & 31); }
    // Does every lane of this warp have all its vectors, of whole pairs?
    static __device__ __forceinline__ bool whole(uint32_t n) { return ((threadIdx.x >> 5) + 1) * WARP * N <= n; }
};
__device__ __forceinline__ float element(const F2* v, int j) { return j & 1 ? hi(v[j / 2]) : lo(v[j / 2]); }

template <typename T> __device__ __forceinline__ F2 pair_of_word(uint32_t w) {
    if constexpr (IsBf16<T>::value) return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w)); return pair(f.x, f.y); }
}

// The rows of one array on their way through the ring. `row`: this thread's first byte of the present row (SHIFT: the warp's first byte);
// `place`: where the warp's stretch of a row is in the ring. ALL: every warp of the group is whole.
template <typename T, int MODE, bool ALL, int NV> struct RingRows {
    using P = Part<T, MODE, NV>;
    static constexpr bool SHIFT = P::SHIFT;
    static constexpr int PIECES = P::STRETCH / 512;                   // rounds of 32 pieces that cover a stretch which begins on 16 bytes
    const char* row;
    uint64_t step, ahead;                                             // bytes to the group's next row, and to the one that is fetched
    uint32_t n, vecs, bytes;                                          // elements and vectors of a row, bytes of the warp's stretch
    bool whole;
    uintptr_t first, behind;                                          // SHIFT: the array's first byte and the one behind its last
    __device__ __forceinline__ RingRows(const void* p, uint64_t stride, uint32_t rows, uint32_t elements, uint32_t r, uint32_t row_step, int rows_ahead)
        : step(row_step * stride * sizeof(T)), ahead(rows_ahead * step), n(elements), vecs((elements + P::N - 1) / P::N), whole(ALL || P::whole(elements)) {
        const uint32_t begin = (threadIdx.x >> 5) * P::STRETCH;
        row = static_cast<const char*>(p) + r * stride * sizeof(T) + begin + (SHIFT ? 0u : (threadIdx.x & 31) * 16u);
        if (SHIFT) {
            bytes = whole ? P::STRETCH : n * (uint32_t)sizeof(T) - begin;
            first = reinterpret_cast<uintptr_t>(p);
            behind = first + ((uint64_t)(rows - 1) * stride + elements) * sizeof(T);
        }
    }
    __device__ __forceinline__ void next() { row += step; }
    // Copies this warp's stretch that begins (SHIFT; else this thread's part of it) at `from`.
    __device__ __forceinline__ void fetch(char* place, const char* from) const {
        const uint32_t lane = threadIdx.x & 31, dst = (uint32_t)__cvta_generic_to_shared(place) + lane * 16u;
        if constexpr (!SHIFT) {
            if (ALL || whole) {
#pragma unroll
                for (int i = 0; i < NV; ++i) copy_async_16(dst + i * 512, from + i * 512);
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (P::first_vector() + i * 32 < vecs) copy_async_16(dst + i * 512, from + i * 512);
            }
        } else {
            const uint32_t pieces = (((uint32_t)reinterpret_cast<uintptr_t>(from) & 15u) + bytes + 15) / 16;
            const uintptr_t begin = reinterpret_cast<uintptr_t>(from) & ~(uintptr_t)15;
            if (begin < first || begin + pieces * 16u > behind) { fetch_edge(place, begin, pieces); return; }
            const char* at = reinterpret_cast<const char*>(begin) + lane * 16u;
            if (whole) {
#pragma unroll
                for (int i = 0; i < PIECES; ++i) copy_async_16(dst + i * 512, at + i * 512);
                if (lane + PIECES * 32 < pieces) copy_async_16(dst + PIECES * 512, at + PIECES * 512);
            } else {
#pragma unroll
                for (int i = 0; i <= PIECES; ++i)
                    if (lane + i * 32 < pieces) copy_async_16(dst + i * 512, at + i * 512);
            }
        }
    }
    // The same at the array's first and last row.
    __device__ __noinline__ void fetch_edge(char* place, uintptr_t begin, uint32_t pieces) const {
        for (uint32_t q = threadIdx.x & 31; q < pieces; q += 32) {
            const uintptr_t at = begin + q * 16u;
            if (at >= first && at + 16 <= behind) copy_async_16((uint32_t)__cvta_generic_to_shared(place) + q * 16u, reinterpret_cast<const void*>(at));
            else
                for (uint32_t e = 0; e < 16; e += sizeof(T))
                    if (at + e >= first && at + e < behind) *reinterpret_cast<T*>(place + q * 16u + e) = *reinterpret_cast<const T*>(at + e);
        }
    }
    // This thread's elements of the row that came from `from`; zeros behind its end.
    template <bool WHOLE> __device__ __forceinline__ void read_as(F2* v, const char* place, const char* from) const {
        const uint32_t lane = threadIdx.x & 31, mis = SHIFT ? (uint32_t)reinterpret_cast<uintptr_t>(from) & 15u : 0u;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = P::first_vector() + i * 32;
            const bool in = WHOLE || q < vecs;
            if constexpr (!SHIFT) {
                const uint4 w = in ? reinterpret_cast<const uint4*>(place)[i * 32 + lane] : make_uint4(0u, 0u, 0u, 0u);
                if constexpr (sizeof(T) == 4) {
                    v[2 * i] = pair(__uint_as_float(w.x), __uint_as_float(w.y));
                    v[2 * i + 1] = pair(__uint_as_float(w.z), __uint_as_float(w.w));
                } else {
                    v[4 * i] = pair_of_word<T>(w.x); v[4 * i + 1] = pair_of_word<T>(w.y);
                    v[4 * i + 2] = pair_of_word<T>(w.z); v[4 * i + 3] = pair_of_word<T>(w.w);
                }
            } else if constexpr (sizeof(T) == 4) {
                const float x = in ? reinterpret_cast<const float*>(place + mis)[i * 32 + lane] : 0.f;
                v[i / 2] = i & 1 ? pair(lo(v[i / 2]), x) : pair(x, 0.f);
            } else {
                const uint32_t* w = reinterpret_cast<const uint32_t*>(place + (mis & 12u)) + (i * 32 + lane);
                uint32_t x = 0u;
                if (in) {
                    x = w[0];
                    if constexpr (MODE == kOdd) {
                        x = __funnelshift_r(x, w[1], (mis & 2u) * 8u);
                        if (!WHOLE && q == n / 2) x &= 0xFFFFu;       // an odd row's last element stands alone
                    }
                }
                v[i] = pair_of_word<T>(x);
            }
        }
    }
    __device__ __forceinline__ void read(F2* v, const char* place, const char* from) const { if (ALL || whole) read_as<true>(v, place, from); else read_as<false>(v, place, from); }
};

// A thread's results to its columns of a row.
template <typename T, int MODE, int NV, bool WHOLE> __device__ __forceinline__ void write_row_as(T* row, const F2* v, uint32_t n) {
    using P = Part<T, MODE, NV>;
    const bool between = MODE == kOdd && (reinterpret_cast<uintptr_t>(row) & 2u);
    T* at = row + P::first_vector() * P::N;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t q = P::first_vector() + i * 32;
        if (!WHOLE && q * P::N >= n) continue;
        float o[P::N];
#pragma unroll
        for (int j = 0; j < P::N; ++j) o[j] = element(v, i * P::N + j);
        if (MODE == kOdd && (between || (!WHOLE && q == n / 2))) {
            at[i * 64] = from_f32<T>(o[0]);
            if (WHOLE || q != n / 2) at[i * 64 + 1] = from_f32<T>(o[1 % P::N]);
        } else Pack<T, P::VB>::store(at + i * 32 * P::N, o);
    }
}
template <typename T, int MODE, bool ALL, int NV> __device__ __forceinline__ void write_row(T* row, const F2* v, uint32_t n, bool whole) {
    if (ALL || whole) write_row_as<T, MODE, NV, true>(row, v, n); else write_row_as<T, MODE, NV, false>(row, v, n);
}

// A thread's weights; `other` where there are none or no columns.
template <typename T, typename W, int MODE, int NV> __device__ __forceinline__ void read_weights(F2* v, const void* weights, float other, uint32_t n) {
    using P = Part<T, MODE, NV>;
    const W* w = static_cast<const W*>(weights);
    const bool pairs = P::N == 2 && (reinterpret_cast<uintptr_t>(w) & (2 * sizeof(W) - 1)) == 0;
    float f[P::E];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t q = P::first_vector() + i * 32;
#pragma unroll
        for (int j = 0; j < P::N; ++j) f[i * P::N + j] = other;
        if (q * P::N >= n) continue;
        if constexpr (MODE == kAligned || P::N == 1) load_weights<W, P::N>(f + i * P::N, w, q * P::N, other);
        else if (w) {
            if (pairs && (MODE != kOdd || q != n / 2)) {
                if constexpr (sizeof(W) == 4) { const float2 x = *reinterpret_cast<const float2*>(w + 2 * q); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
                else { Pack<W, 4> x; x.load(w + 2 * q); f[2 * i] = x.get(0); f[2 * i + 1] = x.get(1); }
            } else {
                f[2 * i] = to_f32(w[2 * q]);
                if (2 * q + 1 < n) f[2 * i + 1] = to_f32(w[2 * q + 1]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < P::E / 2; ++j) v[j] = pair(f[2 * j], f[2 * j + 1]);
}

// ---- narrow rows (H <= 256): L lanes hold a row, 8 elements each, and a warp 32 / L rows, so that a warp's instructions do not depend on
// how little of it a row would fill (bf16, 262144 rows of 64: 14.4 us against 61.5 with a warp for each row, 4.7 TB/s; 65536 rows of 97 that
// begin between words: 16.3 against 37.5). No ring: a warp has ROUNDS such rounds of rows under way in registers, 24 warps an SM (32 with 64
// registers: bf16 rows of 64 16.4, of 128 32.0 against 28.8). VEC: neighbours in vectors of 16 bytes; else single elements L apart, for rows that begin
// anywhere. Bound by instructions below 128 columns (the two sums' exchanges); at 128 the bytes take 0.72 of the time.
constexpr uint32_t kNarrow = 256, kNarrowWarps = 8, kNarrowBlocks = 3;

template <typename T, bool VEC, int L> struct NarrowPart {
    static constexpr int N = VEC ? 16 / (int)sizeof(T) : 1, NV = 8 / N, VB = N * (int)sizeof(T), ROUNDS = VEC && sizeof(T) == 2 ? 4 : 2;
    static __device__ __forceinline__ uint32_t column(int i) { return (threadIdx.x % L + L * i) * N; }        // of vector i
    static __device__ __forceinline__ void load(Pack<T, VB> (&x)[NV], const T* row, uint32_t n) {
#pragma unroll
        for (int i = 0; i < NV; ++i) { if (column(i) < n) x[i].load(row + column(i)); else x[i].clear(); }
    }
    static __device__ __forceinline__ void numbers(F2* v, const Pack<T, VB> (&x)[NV]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = pair(x[2 * j / N].get(2 * j % N), x[(2 * j + 1) / N].get((2 * j + 1) % N));
    }
    template <typename W> static __device__ __forceinline__ void weights(F2* v, const void* w, float other, uint32_t n) {
        float f[8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < N; ++j) f[i * N + j] = other;
            if (column(i) < n) load_weights<W, N>(f + i * N, static_cast<const W*>(w), column(i), other);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = pair(f[2 * j], f[2 * j + 1]);
    }
    static __device__ __forceinline__ void store(T* row, const F2* v, uint32_t n) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = element(v, j);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (column(i) < n) Pack<T, VB>::store(row + column(i), f + i * N);
    }
    static __device__ __forceinline__ F2 inside(F2 v, int j, uint32_t n) {      // pair j; zeros behind the row's end
        return pair(column(2 * j / N) < n ? lo(v) : 0.f, column((2 * j + 1) / N) < n ? hi(v) : 0.f);
    }
    // Sum over the row's lanes of 8 numbers each.
    static __device__ __forceinline__ float sum(float v) {
#pragma unroll
        for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        return v;
    }
};
__device__ __forceinline__ float sum_of_8(const F2* v) { const F2 s = add(add(v[0], v[1]), add(v[2], v[3])); return lo(s) + hi(s); }

template <typename T, typename W, bool VEC, int L>
__global__ void __launch_bounds__(kNarrowWarps * 32, kNarrowBlocks) norm_forward_narrow_kernel(NormArgs a) {
    using P = NarrowPart<T, VEC, L>;
    constexpr int U = P::ROUNDS, PER = 32 / L;
    const uint32_t sub = threadIdx.x % 32 / L;
    const float inv = 1.f / (float)a.H;
    F2 g[4], b[4];
    P::template weights<W>(g, a.gamma, 1.f, a.H);
    P::template weights<W>(b, a.beta, 0.f, a.H);
    const uint64_t step = (uint64_t)gridDim.x * kNarrowWarps * U * PER;
    for (uint64_t r = ((uint64_t)blockIdx.x * kNarrowWarps + threadIdx.x / 32) * U * PER + sub; r - sub < a.rows; r += step) {
        Pack<T, P::VB> in[U][P::NV];
#pragma unroll
        for (int u = 0; u < U; ++u) P::load(in[u], static_cast<const T*>(a.x) + (r + u * PER) * a.x_stride, r + u * PER < a.rows ? a.H : 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            F2 x[4], s[4];
            P::numbers(x, in[u]);
            const float mean = P::sum(sum_of_8(x)) * inv;
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[j] = P::inside(add(x[j], twice(-mean)), j, a.H); s[j] = mul(x[j], x[j]); }
            const float rstd = inverse_root(P::sum(sum_of_8(s)) * inv + a.eps);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fma(mul(x[j], twice(rstd)), g[j], b[j]);
            const uint64_t row = r + u * PER;
            if (row >= a.rows) continue;
            P::store(static_cast<T*>(a.y) + row * a.y_stride, x, a.H);
            if (threadIdx.x % L == 0) {
                if (a.mean_out) a.mean_out[row] = mean;
                if (a.rstd_out) a.rstd_out[row] = rstd;
            }
        }
    }
}
template <typename T, typename W, bool VEC, int L> static cudaError_t forward_narrow(const NormArgs& a, int sms, cudaStream_t st) {
    const uint64_t each = kNarrowWarps * NarrowPart<T, VEC, L>::ROUNDS * (32 / L), blocks = (a.rows + each - 1) / each, cap = (uint64_t)sms * kNarrowBlocks;
    norm_forward_narrow_kernel<T, W, VEC, L><<<(uint32_t)(blocks < cap ? blocks : cap), kNarrowWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T, typename W, bool VEC> static cudaError_t forward_narrow(const NormArgs& a, int sms, cudaStream_t st) {
    if (a.H <= 32) return forward_narrow<T, W, VEC, 4>(a, sms, st);
    if (a.H <= 64) return forward_narrow<T, W, VEC, 8>(a, sms, st);
    if (a.H <= 128) return forward_narrow<T, W, VEC, 16>(a, sms, st);
    if constexpr (VEC && sizeof(T) == 2) return cudaErrorNotSupported;          // not called
    else return forward_narrow<T, W, VEC, 32>(a, sms, st);
}

// blockDim = (G, groups in the block). A group takes R rows at a time: two rows share the barriers, and one's latencies hide the other's.
// gamma and beta wait in shared memory, each thread's own where it left them: as registers they would cost a block of three.
// Bound by memory where rows are many (bf16, 32768 rows of 4096: 88 us, 6.1 TB/s, 0.93 of a copy; the instructions take 54 % of the issue
// slots), by the chain of one pair of rows where blocks have few (f16, 5003 rows of 1367 that begin between words: 12.3 us, 2.2 TB/s).
template <typename T, typename W, int MODE, bool ALL, int NV, int R, int D, int MAXT>
__global__ void __launch_bounds__(MAXT, 768 / MAXT) norm_forward_kernel(NormArgs a) {
    using P = Part<T, MODE, NV>;
    constexpr int H2 = P::E / 2;
    extern __shared__ uint4 ring_memory[];
    __shared__ Scratch scratch;
    uint32_t turn = 0;
    const uint32_t bytes = blockDim.x / 32 * P::PLACE;               // a row in the ring
    char* ring = reinterpret_cast<char*>(ring_memory) + threadIdx.y * D * R * bytes + (threadIdx.x >> 5) * P::PLACE;
    float4* weights = reinterpret_cast<float4*>(reinterpret_cast<char*>(ring_memory) + blockDim.y * D * R * bytes) + threadIdx.x;
    const float inv = 1.f / (float)a.H;
    const uint32_t step = gridDim.x * blockDim.y * R, r0 = (blockIdx.x * blockDim.y + threadIdx.y) * R;
    RingRows<T, MODE, ALL, NV> in(a.x, a.x_stride, a.rows, a.H, r0, step, D - 1);
    const uint64_t x_next = a.x_stride * sizeof(T);                  // bytes to the next row
    T* y = static_cast<T*>(a.y) + r0 * a.y_stride;
    const auto fetch = [&](uint32_t r, char* place, const char* from) {
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (r + k < a.rows) in.fetch(place + k * bytes, from + k * x_next);
        copies_end_batch();
    };
    uint32_t fetched = r0, put = 0, take = 0;
#pragma unroll
    for (int d = 0; d < D - 1; ++d) {
        fetch(fetched, ring + put, in.row + d * in.step);
        fetched += step; put += R * bytes;                           // rows + grid stay below 2^32
    }
    if (threadIdx.y == 0) {
        F2 g[H2], b[H2];
        read_weights<T, W, MODE, NV>(g, a.gamma, 1.f, a.H);
        read_weights<T, W, MODE, NV>(b, a.beta, 0.f, a.H);
#pragma unroll
        for (int j = 0; j < H2 / 2; ++j) {
            weights[2 * j * blockDim.x] = make_float4(lo(g[2 * j]), hi(g[2 * j]), lo(g[2 * j + 1]), hi(g[2 * j + 1]));
            weights[(2 * j + 1) * blockDim.x] = make_float4(lo(b[2 * j]), hi(b[2 * j]), lo(b[2 * j + 1]), hi(b[2 * j + 1]));
        }
    }
    clear_scratch(scratch);
    for (uint32_t r = r0; r < a.rows; r += step) {
        copies_wait<D - 2>();
        if (P::SHIFT) __syncwarp();
        F2 x[R][H2];
        float mean[R], rstd[R];
#pragma unroll
        for (int k = 0; k < R; ++k) in.read(x[k], ring + take + k * bytes, in.row + k * x_next);
        fetch(fetched, ring + put, in.row + in.ahead);
        fetched += step;
        put = take;
        take = take + R * bytes == D * R * bytes ? 0 : take + R * bytes;
        in.next();
#pragma unroll
        for (int k = 0; k < R; ++k) {
            F2 s = x[k][0];
#pragma unroll
            for (int j = 1; j < H2; ++j) s = add(s, x[k][j]);
            mean[k] = lo(s) + hi(s);
        }
        group_sums(mean, scratch, turn);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            mean[k] *= inv;
#pragma unroll
            for (int j = 0; j < H2; ++j) x[k][j] = add(x[k][j], twice(-mean[k]));
            if (!ALL && !in.whole) {                                 // nothing behind the row's end
#pragma unroll
                for (int j = 0; j < H2; ++j) {
                    const uint32_t c = P::N == 1 ? P::first_vector() + 2 * j * 32 : (P::first_vector() + 2 * j / P::N * 32) * P::N + 2 * j % P::N;
                    if (c + (P::N == 1 ? 32 : 1) >= a.H) x[k][j] = pair(c < a.H ? lo(x[k][j]) : 0.f, 0.f);
                }
            }
            F2 s = mul(x[k][0], x[k][0]);
#pragma unroll
            for (int j = 1; j < H2; ++j) s = fma(x[k][j], x[k][j], s);
            rstd[k] = lo(s) + hi(s);
        }
        group_sums(rstd, scratch, turn);
#pragma unroll
        for (int k = 0; k < R; ++k) rstd[k] = inverse_root(rstd[k] * inv + a.eps);
#pragma unroll
        for (int j = 0; j < H2 / 2; ++j) {
            const float4 g = weights[2 * j * blockDim.x], b = weights[(2 * j + 1) * blockDim.x];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                x[k][2 * j] = fma(mul(x[k][2 * j], twice(rstd[k])), pair(g.x, g.y), pair(b.x, b.y));
                x[k][2 * j + 1] = fma(mul(x[k][2 * j + 1], twice(rstd[k])), pair(g.z, g.w), pair(b.z, b.w));
            }
        }
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k == 0 || r + k < a.rows) {
                write_row<T, MODE, ALL, NV>(y + k * a.y_stride, x[k], a.H, in.whole);
                if (threadIdx.x == 0) {
                    if (a.mean_out) a.mean_out[r + k] = mean[k];
                    if (a.rstd_out) a.rstd_out[r + k] = rstd[k];
                }
            }
        y += step * a.y_stride;
    }
}

// blockDim = (G, groups in the block); a group of threads walks the rows of one RowWalk. The weight gradients cost no traffic of
// their own beyond the slots, but 48 registers: 16 warps an SM, each of which waits for a row's chain (ring, two sums over the group, row)
// half of the time. bf16, 32768 rows of 4096 over 64 processes: 135-140 us with the messages, 5.8-6.0 TB/s, 0.88-0.91 of a copy; 8191 rows of 2050
// over ragged processes: 40 us, of which 10 are beginnings and ends (the holder of the first row, the last slot, the second kernel).
template <typename T, typename W, int MODE, bool ALL, int NV, int D>
__global__ void __launch_bounds__(kMaxGroup) norm_backward_kernel(NormArgs a) {
    using P = Part<T, MODE, NV>;
    constexpr int H2 = P::E / 2;
    extern __shared__ uint4 ring_memory[];
    __shared__ Scratch scratch;
    uint32_t turn = 0;
    const uint32_t bytes = blockDim.x / 32 * P::PLACE, group = blockIdx.x * blockDim.y + threadIdx.y;
    char* ring = reinterpret_cast<char*>(ring_memory) + threadIdx.y * D * 2 * bytes + (threadIdx.x >> 5) * P::PLACE;
    later_kernel_may_start();
    clear_scratch(scratch);
    if (group >= a.groups) return;                                   // whole warps, and in blocks of one group nobody
    RowWalk walk(a, group);
    RingRows<T, MODE, ALL, NV> xs(a.x, a.x_stride, a.rows, a.H, walk.r0, 1, D - 1), ys(a.dy, a.dy_stride, a.rows, a.H, walk.r0, 1, D - 1);
    T* dx = static_cast<T*>(a.dx) + walk.r0 * a.dx_stride;
    const float inv = 1.f / (float)a.H;
    uint32_t put = 0, take = 0;
#pragma unroll
    for (int d = 0; d < D - 1; ++d) {
        if (walk.r0 + d < walk.r1) { xs.fetch(ring + put, xs.row + d * xs.step); ys.fetch(ring + put + bytes, ys.row + d * ys.step); }
        copies_end_batch();
        put += 2 * bytes;
    }
    float nmean = 0.f, nrstd = 0.f;
    if (walk.r0 < walk.r1) { nmean = a.mean[walk.r0]; nrstd = a.rstd[walk.r0]; }
    F2 g[H2], dg[H2], db[H2];
    read_weights<T, W, MODE, NV>(g, a.gamma, 1.f, a.H);
#pragma unroll
    for (int j = 0; j < H2; ++j) dg[j] = db[j] = twice(0.f);
    const auto leave = [&](bool direct) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q = P::first_vector() + i * 32;
            if (!ALL && q * P::N >= a.H) continue;
            float x[P::N], y[P::N];
#pragma unroll
            for (int j = 0; j < P::N; ++j) { x[j] = element(dg, i * P::N + j); y[j] = element(db, i * P::N + j); }
            if (direct) store_message<P::N>(a, walk.p, q * P::N, x, y);
            else if (MODE == kOdd && q == a.H / 2) store_slot<1>(a, walk.slot(), q * 2, x, y);
            else store_slot<P::N>(a, walk.slot(), q * P::N, x, y);
        }
    };
    uint32_t weights_from = a.direct ? 0 : ~0u, weights_to = ~0u;    // the rows that count for the present process
    if (a.slots) { walk.find(); weights_from = walk.start; weights_to = walk.end; }
    for (uint32_t r = walk.r0; r < walk.r1; ++r) {
        copies_wait<D - 2>();
        if (P::SHIFT) __syncwarp();
        F2 x[H2], dy[H2];
        xs.read(x, ring + take, xs.row);
        ys.read(dy, ring + take + bytes, ys.row);
        if (r + (D - 1) < walk.r1) { xs.fetch(ring + put, xs.row + xs.ahead); ys.fetch(ring + put + bytes, ys.row + ys.ahead); }
        copies_end_batch();
        put = take;
        take = take + 2 * bytes == D * 2 * bytes ? 0 : take + 2 * bytes;
        xs.next(); ys.next();
        const float mean = nmean, rstd = nrstd;
        if (r + 1 < walk.r1) { nmean = a.mean[r + 1]; nrstd = a.rstd[r + 1]; }
        if (r >= weights_to) {
            if (walk.any) leave(false);
            walk.go_to(r);
#pragma unroll
            for (int j = 0; j < H2; ++j) dg[j] = db[j] = twice(0.f);
            weights_from = walk.start; weights_to = walk.end;
        }
        const bool counts = r >= weights_from;
        walk.any |= counts;
#pragma unroll
        for (int j = 0; j < H2; ++j) x[j] = mul(add(x[j], twice(-mean)), twice(rstd));        // behind the row's end dy = 0 adds nothing
        if (counts) {
#pragma unroll
            for (int j = 0; j < H2; ++j) { dg[j] = fma(dy[j], x[j], dg[j]); db[j] = add(db[j], dy[j]); }
        }
        if (!a.dx) continue;
        F2 s1 = twice(0.f), s2 = twice(0.f);
#pragma unroll
        for (int j = 0; j < H2; ++j) { dy[j] = mul(dy[j], g[j]); s1 = add(s1, dy[j]); s2 = fma(dy[j], x[j], s2); }
        const float2 s = group_sum(make_float2(lo(s1) + hi(s1), lo(s2) + hi(s2)), scratch, turn);
        const F2 c1 = twice(-s.x * inv * rstd), c2 = twice(-s.y * inv * rstd);
#pragma unroll
        for (int j = 0; j < H2; ++j) x[j] = fma(dy[j], twice(rstd), fma(x[j], c2, c1));
        write_row<T, MODE, ALL, NV>(dx, x, a.H, xs.whole);
        dx += a.dx_stride;
    }
    if (a.slots && walk.any) leave(false);
    if (a.direct) {
        leave(true);                                                 // and the last message's fill
        for (uint32_t h = a.H + threadIdx.x; h < (a.H + a.k - 1) / a.k * a.k; h += blockDim.x) {
            const uint64_t o = ((uint64_t)(h / a.k) * a.P + walk.p) * a.k + h % a.k;
            if (a.dgamma) a.dgamma[o] = 0.f;
            if (a.dbeta) a.dbeta[o] = 0.f;
        }
    }
}

// Narrow rows (see the forward pass). blockDim = (32, 4); a warp walks the rows of one RowWalk, 32 / L at a time: the lanes of a row that the
// present process does not hold leave the sums alone, and before the sums are left they are added over the warp's rows. bf16, 262144 rows
// of 64 over 64 processes: 26.7 us (3.9 TB/s) against 107 with a warp for each row; 65536 of 97 that begin between words: 20.5 (24.8 over ragged processes) against 57.
template <typename T, typename W, bool VEC, int L> __global__ void __launch_bounds__(128, 4) norm_backward_narrow_kernel(NormArgs a) {
    using P = NarrowPart<T, VEC, L>;
    constexpr int U = P::ROUNDS;
    constexpr uint32_t PER = 32 / L;
    const uint32_t sub = threadIdx.x / L, group = blockIdx.x * blockDim.y + threadIdx.y;
    later_kernel_may_start();
    if (group >= a.groups) return;                                   // whole warps
    RowWalk walk(a, group);
    const float inv = 1.f / (float)a.H;
    F2 g[4], dg[4], db[4];
    P::template weights<W>(g, a.gamma, 1.f, a.H);
#pragma unroll
    for (int j = 0; j < 4; ++j) dg[j] = db[j] = twice(0.f);
    const auto leave = [&](bool direct) {
        float x[8], y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = element(dg, j); y[j] = element(db, j);
#pragma unroll
            for (int o = L; o < 32; o *= 2) { x[j] += __shfl_xor_sync(0xFFFFFFFFu, x[j], o); y[j] += __shfl_xor_sync(0xFFFFFFFFu, y[j], o); }
        }
        if (sub) return;
#pragma unroll
        for (int i = 0; i < P::NV; ++i) {
            if (P::column(i) >= a.H) continue;
            if (direct) store_message<P::N>(a, walk.p, P::column(i), x + i * P::N, y + i * P::N);
            else store_slot<P::N>(a, walk.slot(), P::column(i), x + i * P::N, y + i * P::N);
        }
    };
    uint32_t from = a.direct ? 0 : ~0u, to = ~0u;                    // the rows that count for the present process
    if (a.slots) { walk.find(); from = walk.start; to = walk.end; }
    for (uint64_t r = walk.r0; r < walk.r1; r += U * PER) {
        Pack<T, P::VB> xs[U][P::NV], ys[U][P::NV];
        float mean[U], rstd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t row = r + u * PER + sub;
            const bool in = row < walk.r1;
            P::load(xs[u], static_cast<const T*>(a.x) + row * a.x_stride, in ? a.H : 0);
            P::load(ys[u], static_cast<const T*>(a.dy) + row * a.dy_stride, in ? a.H : 0);
            mean[u] = in ? a.mean[row] : 0.f;
            rstd[u] = in ? a.rstd[row] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t base = r + u * PER, row = base + sub, stop = base + PER < walk.r1 ? base + PER : walk.r1;
            if (base >= walk.r1) break;
            F2 x[4], dy[4];
            P::numbers(x, xs[u]);
            P::numbers(dy, ys[u]);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = mul(add(x[j], twice(-mean[u])), twice(rstd[u]));      // behind the row's end dy = 0 adds nothing
            while (true) {
                if (row >= from && row < to && row < stop) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) { dg[j] = fma(dy[j], x[j], dg[j]); db[j] = add(db[j], dy[j]); }
                }
                walk.any |= from < stop && to > base;
                if (to >= stop) break;
                if (walk.any) leave(false);
                walk.go_to(to);
#pragma unroll
                for (int j = 0; j < 4; ++j) dg[j] = db[j] = twice(0.f);
                from = walk.start; to = walk.end;
            }
            if (!a.dx) continue;
            F2 s2[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) { dy[j] = mul(dy[j], g[j]); s2[j] = mul(dy[j], x[j]); }
            const float c = rstd[u] * inv;
            const F2 c1 = twice(-P::sum(sum_of_8(dy)) * c), c2 = twice(-P::sum(sum_of_8(s2)) * c);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fma(dy[j], twice(rstd[u]), fma(x[j], c2, c1));
            if (row < stop) P::store(static_cast<T*>(a.dx) + row * a.dx_stride, x, a.H);
        }
    }
    if (a.slots && walk.any) leave(false);
    if (a.direct) {
        leave(true);                                                 // and the last message's fill
        for (uint32_t h = a.H + threadIdx.x; h < (a.H + a.k - 1) / a.k * a.k; h += 32) {
            const uint64_t o = ((uint64_t)(h / a.k) * a.P + walk.p) * a.k + h % a.k;
            if (a.dgamma) a.dgamma[o] = 0.f;
            if (a.dbeta) a.dbeta[o] = 0.f;
        }
    }
}
template <typename T, typename W, bool VEC, int L> static cudaError_t backward_narrow(const NormArgs& a, cudaStream_t st) {
    norm_backward_narrow_kernel<T, W, VEC, L><<<(a.groups + 3) / 4, dim3(32, 4), 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T, typename W, bool VEC> static cudaError_t backward_narrow(const NormArgs& a, cudaStream_t st) {
    if (a.H <= 32) return backward_narrow<T, W, VEC, 4>(a, st);
    if (a.H <= 64) return backward_narrow<T, W, VEC, 8>(a, st);
    if (a.H <= 128) return backward_narrow<T, W, VEC, 16>(a, st);
    if constexpr (VEC && sizeof(T) == 2) return cudaErrorNotSupported;          // not called
    else return backward_narrow<T, W, VEC, 32>(a, st);
}

// Threads that hold a row of H elements, 16 each, and rows of a block of 128 threads where a warp is enough for one.
static inline uint32_t group_threads(uint32_t H) { return (H + 16 * 32 - 1) / (16 * 32) * 32; }
static inline dim3 group_shape(uint32_t vecs, uint32_t nv) {
    const uint32_t g = (vecs + nv * 32 - 1) / (nv * 32) * 32;
    return dim3(g, g == 32 ? 4 : 1);
}

// Blocks of the forward kernel that an SM holds: 768 threads, and their shared memory.
static inline uint32_t forward_per_sm(dim3 block, size_t smem) {
    const uint32_t threads = block.x * block.y, by_threads = threads < 768 ? 768 / threads : 1, by_memory = (uint32_t)(227 * 1024 / (smem + 1536));
    return by_threads < by_memory ? by_threads : by_memory ? by_memory : 1;
}

template <typename K> static cudaError_t allow_shared(K kernel, size_t bytes) {
    return bytes <= 40 * 1024 ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T, typename W, int MODE, bool ALL, int NV, int R, int MAXT> static cudaError_t forward_launch(const NormArgs& a, dim3 block, int sms, cudaStream_t st) {
    using P = Part<T, MODE, NV>;
    constexpr int D = 2;
    const size_t smem = (size_t)block.y * D * R * (block.x / 32) * P::PLACE + (size_t)block.x * P::E * 8;
    const cudaError_t e = allow_shared(norm_forward_kernel<T, W, MODE, ALL, NV, R, D, MAXT>, smem);
    if (e != cudaSuccess) return e;
    const uint32_t blocks = (a.rows + block.y * R - 1) / (block.y * R), cap = (uint32_t)sms * forward_per_sm(block, smem);
    norm_forward_kernel<T, W, MODE, ALL, NV, R, D, MAXT><<<blocks < cap ? blocks : cap, block, smem, st>>>(a);
    return cudaGetLastError();
}
// Two rows at a time where that still leaves every SM its blocks.
template <typename T, typename W, int MODE, bool ALL, int NV> static cudaError_t forward_shape(const NormArgs& a, dim3 block, int sms, cudaStream_t st) {
    const bool two = a.rows >= 2u * sms * forward_per_sm(block, 0) * block.y;
    if (NV == 1 || block.x <= 256)                                   // NV = 1: one warp
        return two ? forward_launch<T, W, MODE, ALL, NV, 2, 256>(a, block, sms, st) : forward_launch<T, W, MODE, ALL, NV, 1, 256>(a, block, sms, st);
    if constexpr (NV > 1) {
        if (two && block.x <= 384) return forward_launch<T, W, MODE, ALL, NV, 2, 384>(a, block, sms, st);
        return two ? forward_launch<T, W, MODE, ALL, NV, 2, kMaxGroup>(a, block, sms, st) : forward_launch<T, W, MODE, ALL, NV, 1, kMaxGroup>(a, block, sms, st);
    }
    return cudaErrorNotSupported;
}
template <typename T, typename W, int MODE, int NV> static cudaError_t forward_run(const NormArgs& a, int sms, cudaStream_t st) {
    using P = Part<T, MODE, NV>;
    const dim3 block = group_shape((a.H + P::N - 1) / P::N, NV);
    if constexpr (MODE == kAligned)
        if (a.H == NV * P::N * block.x) return forward_shape<T, W, MODE, true, NV>(a, block, sms, st);
    return forward_shape<T, W, MODE, false, NV>(a, block, sms, st);
}

// cudaErrorNotSupported: the row does not fit.
template <typename T, typename W> static cudaError_t forward_rows(const NormArgs& a, uint32_t v, int sms, cudaStream_t st) {
    constexpr int e = sizeof(T);
    if (a.H > 16 * kMaxGroup) return cudaErrorNotSupported;
    // Narrow: bf16, 65536 rows of 256 on 16 bytes take 12.4 us by way of the ring against 15.1, all else is faster without it.
    if constexpr (e == 2)
        if (v == 16 && a.H > kNarrow / 2 && a.H <= kNarrow) return forward_run<T, W, kAligned, 1>(a, sms, st);
    if (a.H <= kNarrow) return v == 16 ? forward_narrow<T, W, true>(a, sms, st) : forward_narrow<T, W, false>(a, sms, st);
    if (v == 16) return forward_run<T, W, kAligned, e>(a, sms, st);
    if constexpr (e == 2)
        if (v == 2) return forward_run<T, W, kOdd, 8>(a, sms, st);
    return forward_run<T, W, kWords, 4 * e>(a, sms, st);
}

template <typename T, typename W, int MODE, bool ALL, int NV, int D> static cudaError_t backward_launch(const NormArgs& a, dim3 block, cudaStream_t st) {
    using P = Part<T, MODE, NV>;
    const size_t smem = (size_t)block.y * D * 2 * (block.x / 32) * P::PLACE;
    const cudaError_t e = allow_shared(norm_backward_kernel<T, W, MODE, ALL, NV, D>, smem);
    if (e != cudaSuccess) return e;
    norm_backward_kernel<T, W, MODE, ALL, NV, D><<<(a.groups + block.y - 1) / block.y, block, smem, st>>>(a);
    return cudaGetLastError();
}
template <typename T, typename W, int MODE, int NV, int D> static cudaError_t backward_run(const NormArgs& a, cudaStream_t st) {
    using P = Part<T, MODE, NV>;
    const dim3 block = group_shape((a.H + P::N - 1) / P::N, NV);
    if constexpr (MODE == kAligned)
        if (a.H == NV * P::N * block.x) return backward_launch<T, W, MODE, true, NV, D>(a, block, st);
    return backward_launch<T, W, MODE, false, NV, D>(a, block, st);
}

template <typename T, typename W> static cudaError_t backward_rows(const NormArgs& a, uint32_t v, cudaStream_t st) {
    constexpr int e = sizeof(T), D = e == 2 ? 3 : 2;
    if (a.H > 16 * kMaxGroup) return cudaErrorNotSupported;
    if constexpr (e == 2)                                            // as in the forward pass: 25.7 us against 28.3 over 64 processes
        if (v == 16 && a.H > kNarrow / 2 && a.H <= kNarrow) return backward_run<T, W, kAligned, 1, D>(a, st);
    if (a.H <= kNarrow) return v == 16 ? backward_narrow<T, W, true>(a, st) : backward_narrow<T, W, false>(a, st);
    if (v == 16) return backward_run<T, W, kAligned, e, D>(a, st);
    if constexpr (e == 2)
        if (v == 2) return backward_run<T, W, kOdd, 8, D>(a, st);
    return backward_run<T, W, kWords, 4 * e, D>(a, st);
}

}  // namespace ftc
