// Log probabilities of given tokens, entropy and top alternatives under rows of logits, and the logits' gradient.
//
// Forward: one pass over a row. A lane keeps the largest logit m that it has seen, s = sum(2^d) and t = sum(d 2^d) with d = c x - c m,
// c = scale * log2(e); where a larger one comes, s and t are moved to it. Lanes, warps and blocks are joined the same way; then
//   lse = scale m + ln s,   entropy = ln s - ln 2 * t / s,   logprob = scale (x[token] - m) - ln s.
// The rounding of c m is the same in all terms and is taken out of ln s and t at the end (up to sizes of 1e8; beyond, see below). Bound by memory and by the 16 powers that an SM
// makes a cycle (0.7 of what 16-bit logits need); seven instructions an element (8192 rows of 65536). Logits below -1e30 count as that, so that no infinity meets a
// zero; a row whose largest c m is beyond 1e8 either way, but not -infinity (all of it masked by the type's lowest value, say) is done again with
// c (x - m), element by element.
// Rows are divided over the blocks of a cluster where there are few. 8192 rows of 65536 in bf16: 195 to 207 us by box, 5.2 to 5.5 TB/s; 8 rows of 131072: 10 us.
//
// Top alternatives: the lanes' largest logits are at hand after the pass. The n-th largest of them (its upper 16 bits, found bit by bit by counting
// lanes) is a bound that n elements reach, and about as many do (lanes hold V / 256 elements each): only the lanes that reach it look through their elements again, what reaches the bound is listed
// and ranked by counting. A list that would be too long (equal logits, rows with few finite ones) is left: then warps keep their best 32 in
// their lanes, sorted, and take in what beats the last one that counts.
#include <cooperative_groups.h>
#include "ftc_f32x2.cuh"
#include "ftc_lm.cuh"

namespace ftc {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLeast = -200.f;                                 // 2^-200 is 0 in float32: stands for whatever is smaller
constexpr float kMost = 3.40282346638528859812e38f;              // float32's largest number
constexpr uint32_t kNone = 0xFFFFFFFFu;

__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }

// 16 bytes as numbers.
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void numbers(float* v, uint4 r) {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* v) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void numbers(float* v, uint4 r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    static __device__ __forceinline__ uint4 pack(const float* v) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec<__half> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void numbers(float* v, uint4 r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i])); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
    }
    static __device__ __forceinline__ uint4 pack(const float* v) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

struct Sums { float m, cm, s, t, seen; };                        // m: at least kFloor; cm: c * m, rounded up, so that no d is above 0; seen: the largest logit itself
constexpr float kFloor = -0x1p100f;                              // -1.3e30; its product with c is exact

__device__ __forceinline__ void move_to(Sums& a, float m, float c) {       // m: at least a.m, or NaN
    const float cm = __fmul_ru(m, c), d = fmaxf(a.cm - cm, kLeast), f = exp2_fast(d);
    a.t = fmaf(a.s, d, a.t) * f;
    a.s *= f;
    a.m = m; a.cm = cm;
}
__device__ __forceinline__ void join(Sums& a, Sums b, float c) {
    const float m = max_nan(a.m, b.m);
    move_to(a, m, c);
    move_to(b, m, c);
    a.s += b.s; a.t += b.t;
    a.seen = max_nan(a.seen, b.seen);
}
// The sums of the first LANES lanes together.
template <int LANES> __device__ __forceinline__ Sums joined_lanes(Sums a, float c) {
    float m = a.m;
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) {
        m = max_nan(m, __shfl_xor_sync(kNone, m, o));
        a.seen = max_nan(a.seen, __shfl_xor_sync(kNone, a.seen, o));
    }
    move_to(a, m, c);
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) {
        a.s += __shfl_xor_sync(kNone, a.s, o);
        a.t += __shfl_xor_sync(kNone, a.t, o);
    }
    return a;
}

// 16 bytes: the largest of several such, and pairs of numbers of at least kFloor.
template <typename T> struct Pairs;
template <> struct Pairs<float> {
    static constexpr int N = 2;
    float a, b;
    __device__ __forceinline__ void start() { a = b = -INFINITY; }
    __device__ __forceinline__ void most(uint4 r) {
        a = max_nan(a, max_nan(__uint_as_float(r.x), __uint_as_float(r.y)));
        b = max_nan(b, max_nan(__uint_as_float(r.z), __uint_as_float(r.w)));
    }
    __device__ __forceinline__ float value() const { return max_nan(a, b); }
    static __device__ __forceinline__ void numbers(F2* v, uint4 r) {
        v[0] = pair(fmaxf(__uint_as_float(r.x), kFloor), fmaxf(__uint_as_float(r.y), kFloor));
        v[1] = pair(fmaxf(__uint_as_float(r.z), kFloor), fmaxf(__uint_as_float(r.w), kFloor));
    }
};
__device__ __forceinline__ uint32_t min_u16x2(uint32_t a, uint32_t b) { uint32_t r; asm("min.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
template <> struct Pairs<__nv_bfloat16> {
    static constexpr int N = 4;
    __nv_bfloat162 a;
    __device__ __forceinline__ void start() { a = __floats2bfloat162_rn(-INFINITY, -INFINITY); }
    __device__ __forceinline__ void most(uint4 r) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&r);
        a = __hmax2_nan(a, __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    }
    __device__ __forceinline__ float value() const { return max_nan(__low2float(a), __high2float(a)); }
    static __device__ __forceinline__ void numbers(F2* v, uint4 r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {                            // as whole numbers, negative ones grow with their size: 0xF180 is kFloor
            const uint32_t x = min_u16x2(w[i], 0xF180F180u);
            v[i] = pair(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
        }
    }
};
template <> struct Pairs<__half> {
    static constexpr int N = 4;
    __half2 a;
    __device__ __forceinline__ void start() { a = __floats2half2_rn(-INFINITY, -INFINITY); }
    __device__ __forceinline__ void most(uint4 r) {
        const __half2* h = reinterpret_cast<const __half2*>(&r);
        a = __hmax2_nan(a, __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    }
    __device__ __forceinline__ float value() const { return max_nan(__low2float(a), __high2float(a)); }
    static __device__ __forceinline__ void numbers(F2* v, uint4 r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            v[i] = pair(fmaxf(f.x, kFloor), fmaxf(f.y, kFloor));
        }
    }
};

// The best 32 of a warp, best first, one a lane: a larger word is a better element, equal logits go to the lower index. 0: none.
__device__ __forceinline__ uint64_t word_of(float x, uint32_t index) {
    const uint32_t b = __float_as_uint(x + 0.f), o = b & 0x80000000u ? ~b : b | 0x80000000u;     // -0 is 0
    return (uint64_t)o << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(uint64_t w) {
    const uint32_t o = (uint32_t)(w >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint32_t index_of(uint64_t w) { return ~(uint32_t)w; }
__device__ __forceinline__ void insert(uint64_t& best, uint64_t w, uint32_t lane) {
    const uint32_t at = __popc(__ballot_sync(kNone, best > w));              // sorted: those before it
    const uint64_t up = __shfl_up_sync(kNone, best, 1);
    if (lane == at) best = w;
    else if (lane > at) best = up;
}
// The best 32 of two sorted lists, sorted.
__device__ __forceinline__ uint64_t merged(uint64_t a, uint64_t b, uint32_t lane) {
    const uint64_t r = __shfl_sync(kNone, b, 31 - lane);
    uint64_t x = a > r ? a : r;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const uint64_t y = __shfl_xor_sync(kNone, x, o);
        x = (lane & o) ? (x < y ? x : y) : (x > y ? x : y);
    }
    return x;
}

constexpr uint32_t kListed = 256, kWarpListed = 128;

// A warp's list, as a row is gone through: what an element has to beat.
struct Best {
    uint64_t best;
    float least;
    __device__ __forceinline__ void start() { best = 0; least = -INFINITY; }
    // `count` neighbours of each lane, from `index` on, the largest of them `most`. All lanes together.
    template <typename V> __device__ __forceinline__ void consider(V value, int count, float most, uint32_t index, uint32_t n_top, uint32_t lane) {
        uint32_t lanes = __ballot_sync(kNone, most > least);
        while (lanes) {
            const int src = __ffs(lanes) - 1;
            lanes &= lanes - 1;
            for (int j = 0; j < count; ++j) {
                const float x = __shfl_sync(kNone, value(j), src);
                const uint32_t at = __shfl_sync(kNone, index, src) + j;
                if (x > least) {
                    insert(best, word_of(x, at), lane);
                    const uint64_t w = __shfl_sync(kNone, best, n_top - 1);
                    least = w ? value_of(w) : -INFINITY;
                }
            }
        }
    }
};

// Elements begin .. end-1 of a row: single ones up to the first 16-byte boundary, vectors, single ones behind.
template <typename T> struct Stretch {
    const T* x;
    uint32_t begin, head, vecs, tail, end;
    __device__ __forceinline__ Stretch(const T* row, uint32_t b, uint32_t e) : x(row), begin(b), end(e) {
        constexpr uint32_t N = 16 / sizeof(T);
        const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(x + begin) & 15) / sizeof(T);
        head = min(end, begin + (off ? N - off : 0));
        vecs = (end - head) / N;
        tail = head + vecs * N;
    }
    __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(x + head); }
    __device__ __forceinline__ uint32_t singles() const { return (head - begin) + (end - tail); }
    __device__ __forceinline__ uint32_t single(uint32_t i) const { return i < head - begin ? begin + i : tail + (i - (head - begin)); }
};

template <typename T, bool TOP, uint32_t GROUP> __global__ void __launch_bounds__(GROUP == 32 ? 256 : GROUP, (TOP ? 768 : 1024) / (GROUP == 32 ? 256 : GROUP)) token_logprobs_kernel(LogprobArgs a, uint32_t parts) {
    namespace cg = cooperative_groups;
    constexpr int N = Vec<T>::N;
    constexpr uint32_t kThreads = GROUP == 32 ? 256 : GROUP, kGroups = kThreads / GROUP, kWarps = GROUP / 32;
    __shared__ Sums sums[kThreads / 32];
    __shared__ uint64_t lists[kThreads / 32][32];
    __shared__ Sums joined;
    __shared__ uint64_t joined_list[32];
    constexpr uint32_t kList = GROUP > 32 ? kListed : kWarpListed;
    __shared__ uint64_t listed_of[TOP ? kGroups : 1][TOP ? kList : 1];
    __shared__ uint32_t count_of[kGroups];
    __shared__ uint8_t reaching[TOP ? kThreads / 32 : 1][32];
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, in_group = threadIdx.x % GROUP;
    const uint32_t part = parts > 1 ? cg::this_cluster().block_rank() : 0;
    const float c = a.scale * kLog2e;
    // groups beyond the last row go along with it, so that all threads meet at the barriers
    const uint64_t wanted = (uint64_t)(blockIdx.x / parts) * kGroups + threadIdx.x / GROUP;
    const uint32_t row = (uint32_t)(wanted < a.rows ? wanted : a.rows - 1);
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    const uint32_t share = ((a.V + parts - 1) / parts + 63) & ~63u;
    const uint32_t begin = min(a.V, part * share);
    const Stretch<T> part_of(x, begin, min(a.V, begin + share));
    const uint4* xv = part_of.vectors();
    const uint32_t vecs = part_of.vecs;
    Sums q = {kFloor, kFloor * c, 0.f, 0.f, -INFINITY};
    Best best;
    best.start();
    // the token and its logit, long before they are needed
    int32_t token = -1;
    float token_logit = 0.f;
    if (in_group == 0 && part == 0 && a.logprob) {
        token = token_at(a.tokens, a.token_bits, row, a.V);
        if (token >= 0) token_logit = to_f32(x[token]);
    }
    F2 s2 = twice(0.f), t2 = twice(0.f);
    const F2 c2 = twice(c);
    for (uint32_t i = in_group; i < part_of.singles(); i += GROUP) {
        const float v = to_f32(x[part_of.single(i)]), m = max_nan(q.m, v);
        move_to(q, m, c);
        q.seen = max_nan(q.seen, v);
        const float d = fmaf(fmaxf(v, kFloor), c, -q.cm), e = exp2_fast(d);
        q.s += e;
        q.t = fmaf(d, e, q.t);
    }
    constexpr uint32_t U = 4;
    for (uint32_t i0 = in_group - lane; i0 < vecs; i0 += GROUP * U) {
        uint4 r[U];
        Pairs<T> most;
        most.start();
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * GROUP + lane;
            if (i < vecs) r[u] = __ldg(xv + i);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
            if (i0 + u * GROUP + lane < vecs) most.most(r[u]);
        const float m = most.value();
        q.seen = max_nan(q.seen, m);
        if (!(m <= q.m)) {
            q.s += lo(s2) + hi(s2); q.t += lo(t2) + hi(t2);
            s2 = t2 = twice(0.f);
            move_to(q, max_nan(q.m, m), c);
        }
        const F2 back = twice(-q.cm);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (i0 + u * GROUP + lane >= vecs) continue;
            F2 v[Pairs<T>::N];
            Pairs<T>::numbers(v, r[u]);
#pragma unroll
            for (int j = 0; j < Pairs<T>::N; ++j) {
                const F2 d = fma(v[j], c2, back), e = pair(exp2_fast(lo(d)), exp2_fast(hi(d)));
                s2 = add(s2, e);
                t2 = fma(d, e, t2);
            }
        }
    }
    q.s += lo(s2) + hi(s2); q.t += lo(t2) + hi(t2);
    const float lane_most = q.seen;

    q = joined_lanes<32>(q, c);
    if (GROUP > 32 && lane == 0) sums[warp] = q;
    if (TOP) {
        uint64_t* const listed = listed_of[threadIdx.x / GROUP];
        uint32_t* const counted = &count_of[threadIdx.x / GROUP];
        auto sync = [] { if (GROUP == 32) __syncwarp(); else __syncthreads(); };
        const uint32_t mine = (uint32_t)(word_of(lane_most, 0) >> 48);           // in order, as whole numbers
        uint32_t bound = 0;
#pragma unroll
        for (int bit = 15; bit >= 0; --bit) {
            const uint32_t more = bound | 1u << bit;
            const int reach = GROUP == 32 ? __popc(__ballot_sync(kNone, mine >= more)) : __syncthreads_count(mine >= more);
            if ((uint32_t)reach >= a.top) bound = more;
        }
        if (in_group == 0) *counted = 0;
        sync();
        const bool any = bound <= 0x7Fu;                         // fewer lanes than that have seen a logit above -infinity
        const float least = any ? -INFINITY : value_of((uint64_t)bound << 48 | 0xFFFFFFFFu);
        auto list = [&](float v, uint32_t at) {
            if (v >= least && v > -INFINITY) {
                const uint32_t to = atomicAdd(counted, 1);
                if (to < kList) listed[to] = word_of(v, at);
            }
        };
        if (in_group < part_of.singles()) { const uint32_t at = part_of.single(in_group); list(to_f32(x[at]), at); }
        // the warp's lanes that reach it, and all their vectors one after the other over the warp
        const uint32_t lanes = __ballot_sync(kNone, lane_most >= least && lane_most > -INFINITY), each = (vecs + GROUP - 1) / GROUP;
        if (lanes >> lane & 1u) reaching[warp][__popc(lanes & ((1u << lane) - 1))] = (uint8_t)lane;
        __syncwarp();
        constexpr uint32_t kAtOnce = 4;
        for (uint32_t k0 = 0, all = __popc(lanes) * each; k0 < all; k0 += 32 * kAtOnce) {
            uint4 r[kAtOnce];
            uint32_t at[kAtOnce];
#pragma unroll
            for (uint32_t u = 0; u < kAtOnce; ++u) {
                const uint32_t k = k0 + u * 32 + lane, o = k / each;
                at[u] = k < all ? (in_group - lane) + reaching[warp][o] + (k - o * each) * GROUP : vecs;
                if (at[u] < vecs) r[u] = __ldg(xv + at[u]);
            }
#pragma unroll
            for (uint32_t u = 0; u < kAtOnce; ++u) {
                if (at[u] >= vecs) continue;
                float v[N];
                Vec<T>::numbers(v, r[u]);
#pragma unroll
                for (int j = 0; j < N; ++j) list(v[j], part_of.head + at[u] * N + j);
            }
        }
        sync();
        const uint32_t n = *counted;
        uint64_t* const ranked = lists[warp - in_group / 32];
        if (n <= kList) {                                        // ranked: those among the first 32 have their place
            if (in_group < 32) ranked[in_group] = 0;
            sync();
            for (uint32_t k = in_group; k < n; k += GROUP) {
                const uint64_t w = listed[k];
                uint32_t before = 0;
                for (uint32_t i = 0; i < n; ++i) before += listed[i] > w;
                if (before < 32) ranked[before] = w;
            }
            sync();
            best.best = ranked[lane];
        } else {                                                 // one after the other
            constexpr uint32_t kAhead = 8;
            for (uint32_t i0 = begin + in_group - lane; i0 < part_of.end; i0 += GROUP * kAhead) {
                float v[kAhead], most = -INFINITY;
#pragma unroll
                for (uint32_t k = 0; k < kAhead; ++k) {
                    const uint32_t i = i0 + k * GROUP + lane;
                    v[k] = i < part_of.end ? to_f32(x[i]) : -INFINITY;
                }
#pragma unroll
                for (uint32_t k = 0; k < kAhead; ++k) most = fmaxf(most, v[k]);
                if (!__any_sync(kNone, most > best.least)) continue;
#pragma unroll
                for (uint32_t k = 0; k < kAhead; ++k)
                    best.consider([&](int) { return v[k]; }, 1, v[k], i0 + k * GROUP + lane, a.top, lane);
            }
            if (GROUP > 32) {
                lists[warp][lane] = best.best;
                __syncthreads();
                if (warp == 0)
                    for (uint32_t w = 1; w < kWarps; ++w) best.best = merged(best.best, lists[w][lane], lane);
            }
        }
    }
    if (GROUP > 32) {
        if (!TOP) __syncthreads();
        if (warp == 0) q = joined_lanes<kWarps>(sums[lane % kWarps], c);
        if (parts > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            if (warp == 0) {
                if (lane == 0) joined = q;
                if (TOP) joined_list[lane] = best.best;
            }
            cluster.sync();
            if (part == 0 && warp == 0) {
                for (uint32_t b = 1; b < parts; ++b) {
                    join(q, *cluster.map_shared_rank(&joined, b), c);
                    if (TOP) best.best = merged(best.best, cluster.map_shared_rank(joined_list, b)[lane], lane);
                }
            }
            cluster.sync();                                      // a block's shared memory stays until it has been read
        }
        if (warp || part) return;
    }
    if (wanted >= a.rows) return;

    // one warp has the row now
    float m, ln_s = logf(q.s) - kLn2 * fmaf(q.m, c, -q.cm), mean_d = q.t / q.s - fmaf(q.m, c, -q.cm);      // mean of d, about c m itself
    m = q.seen;
    if (fabsf(m * c) > 1e8f && fabsf(m) < INFINITY) {            // nothing but the type's lowest value, or the like: d = c (x - m), which holds anywhere
        float s = 0.f, t = 0.f;
#pragma unroll 8
        for (uint32_t i = lane; i < a.V; i += 32) {
            const float d = fmaxf((to_f32(x[i]) - m) * c, kLeast), e = exp2_fast(d);
            s += e;
            t = fmaf(d, e, t);
        }
        s = warp_sum(s); t = warp_sum(t);
        ln_s = logf(s); mean_d = t / s;
    }
    const bool bad = isnan(m) || m == INFINITY, empty = m == -INFINITY;
    auto below = [&](float v) { return fmaf(2.f * a.scale, 0.5f * v - 0.5f * m, -ln_s); };      // scale (v - m) - ln s; v - m itself may leave float32
    // scale * m may leave float32: the largest number stands for it then, so that an lse of -infinity is that of an empty row and no other
    const float nan = __int_as_float(0x7FFFFFFF), lse = bad ? nan : empty ? -INFINITY : fminf(fmaxf(fmaf(a.scale, m, ln_s), -kMost), kMost);
    if (lane == 0) {
        if (a.lse) a.lse[row] = lse;
        if (a.entropy) a.entropy[row] = bad ? nan : empty ? 0.f : fmaxf(0.f, ln_s - kLn2 * mean_d);
        if (a.logprob) {
            a.logprob[row] = token < 0 ? 0.f : bad ? nan : empty ? -INFINITY : below(token_logit);
        }
    }
    if (!TOP) return;
    // fewer logits above -infinity than were asked for: the lowest tokens of the others (of a row with NaN or infinity nothing is looked for)
    uint32_t have = bad ? a.top : __popc(__ballot_sync(kNone, best.best != 0));
    for (uint32_t i0 = 0; i0 < a.V && have < a.top; i0 += 32) {
        uint32_t more = __ballot_sync(kNone, i0 + lane < a.V && to_f32(x[min(i0 + lane, a.V - 1)]) == -INFINITY);
        while (more && have < a.top) {
            const uint32_t j = __ffs(more) - 1;
            more &= more - 1;
            if (lane == have) best.best = word_of(-INFINITY, i0 + j);
            ++have;
        }
    }
    if (lane < a.top) {
        const float v = value_of(best.best);
        a.top_logprob[(uint64_t)row * a.top + lane] = bad ? nan : empty ? -INFINITY : below(v);
        a.top_token[(uint64_t)row * a.top + lane] = best.best ? (int32_t)index_of(best.best) : 0;
    }
}

constexpr uint32_t kManyRows = 6, kWarpVectors = 512;
template <typename T, bool TOP, uint32_t GROUP> static cudaError_t forward_of(const LogprobArgs& a, uint32_t parts, cudaStream_t st) {
    constexpr uint32_t kThreads = GROUP == 32 ? 256 : GROUP, kGroups = kThreads / GROUP;
    if (parts == 1) {
        token_logprobs_kernel<T, TOP, GROUP><<<(a.rows + kGroups - 1) / kGroups, kThreads, 0, st>>>(a, 1);
        return cudaGetLastError();
    }
    cudaLaunchAttribute shape{};
    shape.id = cudaLaunchAttributeClusterDimension;
    shape.val.clusterDim.x = parts; shape.val.clusterDim.y = shape.val.clusterDim.z = 1;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3(a.rows * parts); how.blockDim = dim3(kThreads); how.stream = st; how.attrs = &shape; how.numAttrs = 1;
    return cudaLaunchKernelEx(&how, token_logprobs_kernel<T, TOP, GROUP>, a, parts);
}

template <typename T, bool TOP> static cudaError_t forward(const LogprobArgs& a, int sms, cudaStream_t st) {
    const uint32_t vecs = (uint32_t)((uint64_t)a.V * sizeof(T) / 16);
    if (vecs <= 64 || (vecs <= kWarpVectors && a.rows >= 32u * sms)) return forward_of<T, TOP, 32>(a, 1, st);    // a warp for each row
    // Blocks of a cluster share a row while there are SMs without one. Many rows: blocks of 128 threads, so that more rows are on their way
    // while others are joined.
    uint32_t parts = 1;
    while (parts < 8 && (uint64_t)a.rows * parts * 2 <= (uint64_t)sms * 2 && a.V / (parts * 2) >= 4096) parts *= 2;
    if (a.rows >= kManyRows * (uint32_t)sms) return forward_of<T, TOP, 128>(a, 1, st);
    return forward_of<T, TOP, 256>(a, parts, st);
}

cudaError_t launch_token_logprobs(const LogprobArgs& a, int sms, cudaStream_t st) {
    if (a.dtype == FTC_F32) return a.top ? forward<float, true>(a, sms, st) : forward<float, false>(a, sms, st);
    if (a.dtype == FTC_BF16) return a.top ? forward<__nv_bfloat16, true>(a, sms, st) : forward<__nv_bfloat16, false>(a, sms, st);
    return a.top ? forward<__half, true>(a, sms, st) : forward<__half, false>(a, sms, st);
}

// ---- gradient ----
//
// With A = -scale (dlogprob + dentropy * entropy), B = -scale * dentropy and l = scale x - lse, rounded once: p (A + B l), and scale * dlogprob more at
// the token. (A + B' x with lse in A would cancel: lse's size over 2^24 of an error.)
// Bound by memory (8192 rows of 65536 in bf16: 330 to 342 us by box, 6.3 to 6.5 TB/s); twelve instructions an element. A row is written in vectors
// from its own 16-byte boundary on. Where the logits lie otherwise against that boundary (a slice of a padded matrix), a vector is put together from the two that cover it.

// far: lse in float32 is too coarse for the type: half its step, which is p's relative error, is 2^-18 below 2^7 (float32), 2^-14 below 2^11 (float16,
// whose half step is 2^-11), 2^-11 below 2^14 (bfloat16, 2^-8); or B takes the 2^100 that stands for an infinity out of float32.
template <typename T> constexpr float kFarLse = sizeof(T) == 4 ? 0x1p7f : 0x1p14f;
template <> constexpr float kFarLse<__half> = 0x1p11f;
struct RowFactors { float a, b, up, lse; int32_t token; bool zero, far; };

template <typename T> __device__ __forceinline__ RowFactors factors_of(const LogprobArgs& g, uint32_t row) {
    RowFactors f;
    f.token = g.dlogprob ? token_at(g.tokens, g.token_bits, row, g.V) : -1;
    const float given = g.dlogprob ? g.dlogprob[row] : 0.f, up = f.token >= 0 ? given : 0.f, de = g.dentropy ? g.dentropy[row] : 0.f;
    f.lse = g.lse_in[row];
    f.zero = f.lse == -INFINITY;
    f.a = -(g.dentropy ? fmaf(de, g.entropy_in[row], up) : up) * g.scale;
    f.b = -de * g.scale;
    f.up = up * g.scale;
    f.far = fabsf(f.lse) < INFINITY && (fabsf(f.lse) >= kFarLse<T> || fabsf(f.b * g.scale) >= 0x1p26f);
    return f;
}
__device__ __forceinline__ float gradient(const RowFactors& f, float x, float scale) {
    const float v = x < kFloor ? kFloor : x, l = fmaf(v, scale, -f.lse);         // NaN stays
    return f.zero ? 0.f : exp2_fast(l * kLog2e) * fmaf(f.b, l, f.a);
}
// As Pairs' numbers, but NaN stays what it is: the row's lse is NaN then, so no care is needed.
template <typename T> __device__ __forceinline__ uint4 gradients(const RowFactors& f, uint4 r, float scale) {
    constexpr int N = Pairs<T>::N;
    F2 v[N];
    float y[2 * N];
    Pairs<T>::numbers(v, r);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const F2 l = fma(v[j], twice(scale), twice(-f.lse)), d = mul(l, twice(kLog2e)), e = mul(pair(exp2_fast(lo(d)), exp2_fast(hi(d))), fma(twice(f.b), l, twice(f.a)));
        y[2 * j] = f.zero ? 0.f : lo(e);
        y[2 * j + 1] = f.zero ? 0.f : hi(e);
    }
    return Vec<T>::pack(y);
}
// 16 bytes from byte `shift` (1 .. 15) of two vectors on.
__device__ __forceinline__ uint4 joined_at(uint4 a, uint4 b, uint32_t shift) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (shift & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (shift & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    const uint32_t bits = (shift & 3) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

// A far row by one group of threads: its largest logit and sum once more, then scale (dlogprob ([j = token] - p) - dentropy p (log p + entropy)) with
// log p = c (x - m) ln 2 - ln s. A thread reads and writes the same elements. One block has such a row, in three passes: 4096 rows of 65536 in float32
// take 1045 us so, and 322 if none is far (64 of 131072: 134 and 11). Logits whose lse is that large are rare, and exact gradients worth more.
template <typename T, uint32_t GROUP> __device__ __forceinline__ void far_row(const LogprobArgs& g, uint32_t row, const RowFactors& f, const T* x, T* d) {
    __shared__ float parts[2][8];
    const uint32_t in_group = threadIdx.x % GROUP, warp = threadIdx.x / 32;
    const float c = g.scale * kLog2e;
    float m = -INFINITY, s = 0.f;
#pragma unroll 8
    for (uint32_t e = in_group; e < g.V; e += GROUP) m = fmaxf(m, to_f32(x[e]));
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kNone, m, o));
    if (GROUP > 32) {
        if (threadIdx.x % 32 == 0) parts[0][warp] = m;
        __syncthreads();
        for (uint32_t w = 0; w < 8; ++w) m = fmaxf(m, parts[0][w]);
    }
    auto power = [&](float v) { return fmaxf((v - m) * c, kLeast); };
#pragma unroll 8
    for (uint32_t e = in_group; e < g.V; e += GROUP) s += exp2_fast(power(to_f32(x[e])));
    s = warp_sum(s);
    if (GROUP > 32) {
        if (threadIdx.x % 32 == 0) parts[1][warp] = s;
        __syncthreads();
        s = 0.f;
        for (uint32_t w = 0; w < 8; ++w) s += parts[1][w];
    }
    const float ln_s = logf(s), each = 1.f / s, de = g.dentropy ? g.dentropy[row] : 0.f, up = f.token >= 0 ? g.dlogprob[row] : 0.f;
    const float all = fmaf(de, (g.dentropy ? g.entropy_in[row] : 0.f) - ln_s, up) * -g.scale, slope = -g.scale * de * kLn2;
#pragma unroll 8
    for (uint32_t e = in_group; e < g.V; e += GROUP) {
        const float v = power(to_f32(x[e])), y = exp2_fast(v) * each * fmaf(slope, v, all);
        d[e] = from_f32<T>(e == (uint32_t)f.token ? y + f.up : y);
    }
    if (GROUP > 32) __syncthreads();
}

// A unit: up to kPieceVectors vectors of a row for a block (half of that: 358 us in place of 334, double: slower where rows are few), a row for a
// warp (GROUP = 32). Five blocks an SM: 18304 logits a row take 6 % less than with four.
constexpr uint32_t kPieceVectors = 4096;
template <typename T, uint32_t GROUP> __global__ void __launch_bounds__(256, 5) logprobs_backward_kernel(LogprobArgs g, uint32_t pieces, uint32_t each, uint64_t units) {
    constexpr uint32_t N = 16 / sizeof(T), U = 4, kGroups = 256 / GROUP;
    const uint32_t in_group = threadIdx.x % GROUP;
    for (uint64_t unit = (uint64_t)blockIdx.x * kGroups + threadIdx.x / GROUP; unit < units; unit += (uint64_t)gridDim.x * kGroups) {
        const uint32_t row = pieces == 1 ? (uint32_t)unit : (uint32_t)(unit / pieces), piece = pieces == 1 ? 0 : (uint32_t)(unit - (uint64_t)row * pieces);
        const T* const x = static_cast<const T*>(g.logits) + row * g.stride;
        T* const d = static_cast<T*>(g.dlogits) + row * g.dstride;
        const Stretch<T> out(d, 0, g.V);                         // where d has its boundaries
        const uint32_t end = GROUP == 32 ? out.vecs : min(out.vecs, (piece + 1) * each);
        const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(x + out.head) & 15);
        const uint4* const xv = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(x + out.head) - shift);
        uint4* const dv = reinterpret_cast<uint4*>(d + out.head);
        const RowFactors f = factors_of<T>(g, row);
        const uint32_t stores = f.far ? 0 : end;                 // the loads do not wait for it
        const uint32_t at = f.token >= 0 && !f.zero ? (uint32_t)f.token : kNone;
        for (uint32_t i0 = (GROUP == 32 ? 0 : piece * each) + in_group; i0 < end; i0 += GROUP * U) {
            uint4 r[U];
            if (shift) {
#pragma unroll
                for (uint32_t u = 0; u < U; ++u) {
                    const uint32_t i = i0 + u * GROUP;
                    if (i < end) r[u] = joined_at(__ldg(xv + i), __ldg(xv + i + 1), shift);      // the second one holds some of the vector's last element at least
                }
            } else if (g.logits == g.dlogits) {
#pragma unroll
                for (uint32_t u = 0; u < U; ++u)
                    if (i0 + u * GROUP < end) r[u] = xv[i0 + u * GROUP];
            } else {
#pragma unroll
                for (uint32_t u = 0; u < U; ++u)
                    if (i0 + u * GROUP < end) r[u] = __ldg(xv + i0 + u * GROUP);
            }
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint32_t i = i0 + u * GROUP;
                if (i >= stores) continue;
                dv[i] = gradients<T>(f, r[u], g.scale);
                if (at - (out.head + i * N) < N) {               // the token is among them
                    float v[N];
                    Vec<T>::numbers(v, r[u]);
#pragma unroll
                    for (uint32_t j = 0; j < N; ++j)
                        if (out.head + i * N + j == at) d[at] = from_f32<T>(gradient(f, v[j], g.scale) + f.up);
                }
            }
        }
        if (f.far) {
            if (piece == 0) far_row<T, GROUP>(g, row, f, x, d);
            continue;
        }
        if (piece == 0)
            for (uint32_t i = in_group; i < out.singles(); i += GROUP) {
                const uint32_t e = out.single(i);
                const float y = gradient(f, to_f32(x[e]), g.scale);
                d[e] = from_f32<T>(e == at ? y + f.up : y);
            }
    }
}

template <typename T> static cudaError_t backward(const LogprobArgs& g, int sms, cudaStream_t st) {
    // A warp for rows of up to 256 vectors.
    const uint32_t vecs = (uint32_t)(((uint64_t)g.V * sizeof(T) + 15) / 16);
    const bool warps = vecs <= 256;
    const uint32_t pieces = warps ? 1 : (vecs + kPieceVectors - 1) / kPieceVectors;
    const uint32_t each = ((vecs + pieces - 1) / pieces + 255) & ~255u;
    const uint64_t units = (uint64_t)g.rows * pieces, blocks = warps ? (units + 7) / 8 : units, cap = (uint64_t)sms * 256;
    const uint32_t grid = (uint32_t)(blocks < cap ? blocks : cap);
    if (warps) logprobs_backward_kernel<T, 32><<<grid, 256, 0, st>>>(g, pieces, each, units);
    else logprobs_backward_kernel<T, 256><<<grid, 256, 0, st>>>(g, pieces, each, units);
    return cudaGetLastError();
}

cudaError_t launch_token_logprobs_backward(const LogprobArgs& g, int sms, cudaStream_t st) {
    if (g.dtype == FTC_F32) return backward<float>(g, sms, st);
    if (g.dtype == FTC_BF16) return backward<__nv_bfloat16>(g, sms, st);
    return backward<__half>(g, sms, st);
}

}  // namespace ftc
