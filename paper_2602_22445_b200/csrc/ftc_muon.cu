// Orthogonalised updates of many matrices: momentum, then Newton-Schulz steps X <- a X + (b A + c A A) X with A = X X^T, then the weights.
//
// Two kernels take the momentum and lay out X = U / |U| (m x w, m <= w: matrices with more rows than columns transposed), three products a
// step follow, each over all matrices at once:
//   gram   A = X X^T             symmetric: tiles on and below the diagonal, written twice
//   poly   B = b A + c A A       symmetric too (A A = A A^T)
//   apply  X = a X + B X         the last one updates the weights instead
// Operands are float16, held times 2^14: |X| stays below 1.21 after the first step (the largest value of the quintic on 0 .. 1.21), entries of
// A below 1.47 and of B below 2.81, so nothing overflows and numbers down to 2^-28 keep their 11 bits (bfloat16 would keep 8). Diagonals,
// which are the large entries of A and B in late steps, are held apart in float32: with A = D + A', A A = A' A' + D A' + A' D + D D, all but
// the first by elements. Sums are float32 throughout, in tensor memory.
// With `split` every operand is two float16 numbers, the second one what the first leaves over: hi hi + hi lo + lo hi in one sum.
//
// Matrices lie in the workspace in blocks of 128 rows x 64 columns (16 KB), their 16-byte pieces in the order that the tensor cores read
// (piece c of row r at c ^ r % 8): a block is one contiguous copy, whichever way a product reads it, and edges are zeros.
#include "ftc_lm.cuh"

namespace ftc {

constexpr float kQ1 = 3.4445f, kQ3 = -4.7750f, kQ5 = 2.0315f;
constexpr float kUp = 16384.f, kDown = 1.f / 16384.f, kDown2 = kDown * kDown;    // 2^14
constexpr uint32_t kBlockBytes = 128 * 64 * 2;

// The matrix whose run item u is in: first[i] <= u < first[i + 1].
__device__ __forceinline__ uint32_t matrix_of(const uint32_t* first, uint32_t n, uint32_t u) {
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (__ldg(first + mid) <= u) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float element(const void* p, uint32_t dtype, uint64_t i) {
    if (dtype == FTC_F32) return static_cast<const float*>(p)[i];
    if (dtype == FTC_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void set_element(void* p, uint32_t dtype, uint64_t i, float v) {
    if (dtype == FTC_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == FTC_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
// What the gradient is multiplied with: 1 / processes included, 0: not delivered.
__device__ __forceinline__ float share_at(const PlanEntry& t, uint64_t i) {
    if (!t.status) return 1.f;
    const uint64_t q = t.k_shift != 255 ? i >> t.k_shift : (uint32_t)i / t.k;
    const uint2 s = *reinterpret_cast<const uint2*>(t.status + q * FTC_STATUS_WORDS);
    return (s.x & 0xFFu) == FTC_ST_OK && s.y ? 1.f / (float)s.y : 0.f;
}

// ---- momentum ----

__global__ void __launch_bounds__(256) muon_momentum_kernel(MuonArgs a) {
    later_kernel_may_start();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.word = 0;
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!isfinite(scale)) return;
    const uint32_t* first = plan_first(a.plan, a.n, kChunkFirst);
    const uint32_t which = matrix_of(first, a.n, blockIdx.x);
    const PlanEntry& t = plan_entries(a.plan)[which];
    const uint64_t begin = (uint64_t)(blockIdx.x - first[which]) * kMuonChunk;
    const uint32_t left = (uint32_t)min((uint64_t)kMuonChunk, t.n - begin);
    float* m = a.momentum + t.first_block * FTC_STATE_BLOCK + begin;
    double sum = 0;
    uint32_t live = 0;
#pragma unroll 8
    for (uint32_t j = threadIdx.x; j < left; j += 256) {
        const float s = share_at(t, begin + j), old = m[j];
        const float g = element(t.grad, t.grad_dtype, begin + j) * s * scale;
        float now = old, u = old;
        if (s > 0.f) {
            now = fmaf(old, a.mu, g);
            u = a.nesterov ? fmaf(now, a.mu, g) : now;
            m[j] = now;
            live = 1;
        }
        sum = fma((double)u, (double)u, sum);
    }
    __shared__ double sums[8];
    __shared__ uint32_t lives[8];
    sum = warp_sum(sum);
    live = __any_sync(0xFFFFFFFFu, live);
    if (threadIdx.x % 32 == 0) { sums[threadIdx.x / 32] = sum; lives[threadIdx.x / 32] = live; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) { sum += sums[w]; live |= lives[w]; }
        a.sums[blockIdx.x] = make_double2(sum, live ? 1.0 : 0.0);
    }
}

// Where the 16-byte piece c of row r lies in a block.
__device__ __forceinline__ uint32_t piece(uint32_t r, uint32_t c) { return r * 128 + ((c ^ (r & 7)) << 4); }

// One block of 128 x 64 of X.
__global__ void __launch_bounds__(256) muon_layout_kernel(MuonArgs a) {
    wait_for_earlier_kernel();
    later_kernel_may_start();
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!isfinite(scale)) return;
    const uint32_t* first = plan_first(a.plan, a.n, kBlockFirst);
    const uint32_t which = matrix_of(first, a.n, blockIdx.x);
    const PlanEntry& t = plan_entries(a.plan)[which];
    const uint32_t at = blockIdx.x - first[which], bi = at / t.nb, bj = at - bi * t.nb;
    // the norm: all chunks' sums, in the same order in every block
    __shared__ double sums[8], lives[8];
    const uint32_t c0 = plan_first(a.plan, a.n, kChunkFirst)[which], c1 = plan_first(a.plan, a.n, kChunkFirst)[which + 1];
    double sum = 0, live = 0;
    for (uint32_t c = c0 + threadIdx.x; c < c1; c += 256) { const double2 s = a.sums[c]; sum += s.x; live += s.y; }
    sum = warp_sum(sum); live = warp_sum(live);
    if (threadIdx.x % 32 == 0) { sums[threadIdx.x / 32] = sum; lives[threadIdx.x / 32] = live; }
    __syncthreads();
    sum = sums[0]; live = lives[0];
    for (int w = 1; w < 8; ++w) { sum += sums[w]; live += lives[w]; }
    if (at == 0 && threadIdx.x == 0) a.live[which] = live > 0;
    const float inv = (float)((double)kUp / (sqrt(sum) + (double)a.eps));
    const float* m = a.momentum + t.first_block * FTC_STATE_BLOCK;
    __shared__ __align__(16) unsigned char tile[2][kBlockBytes];
#pragma unroll 8
    for (uint32_t e = threadIdx.x; e < 128 * 64; e += 256) {
        const uint32_t r = t.tall ? e % 128 : e / 64, c = t.tall ? e / 128 : e % 64;      // neighbours in memory for neighbouring threads
        const uint32_t i = bi * 128 + r, j = bj * 64 + c;
        float v = 0.f;
        if (i < t.m && j < t.w) {
            const uint64_t q = t.tall ? (uint64_t)j * t.cols + i : (uint64_t)i * t.cols + j;
            v = m[q];
            if (a.nesterov) {
                const float s = share_at(t, q);
                if (s > 0.f) v = fmaf(v, a.mu, element(t.grad, t.grad_dtype, q) * s * scale);
            }
            v *= inv;
        }
        const __half h = __float2half_rn(v);
        const uint32_t to = piece(r, c / 8) + c % 8 * 2;
        *reinterpret_cast<__half*>(tile[0] + to) = h;
        if (a.split) *reinterpret_cast<__half*>(tile[1] + to) = __float2half_rn(v - __half2float(h));
    }
    __syncthreads();
    for (uint32_t s = 0; s <= a.split; ++s) {
        uint4* to = reinterpret_cast<uint4*>(a.x[0] + s * a.x_bytes + (t.x_block + at) * kBlockBytes);
        const uint4* from = reinterpret_cast<const uint4*>(tile[s]);
        for (uint32_t e = threadIdx.x; e < kBlockBytes / 16; e += 256) to[e] = from[e];
    }
}

// ---- products ----
//
// Persistent blocks of eight warps: one thread copies, one issues matrix instructions, four warps read sums out of tensor memory. A tile
// is 128 x 256, its sum 256 columns of tensor memory; there are two, so that one tile is read out while the next is multiplied. A stage
// holds 64 of the inner dimension: 16 KB of the left operand, up to 32 of the right one.

constexpr uint32_t kStages = 4, kStageBytes = 48 * 1024, kOutBytes = 4 * 32 * 33 * 4, kProductThreads = 256;
constexpr uint32_t kProductSmem = kStages * kStageBytes + kOutBytes + 1024 + 256;
enum { kGram, kPoly, kApply, kUpdate };

__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Looks at most 2^22 times (each look may sleep for a while): false if the phase did not end.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < 1u << 22; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}
__device__ __forceinline__ void copy_in(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t how, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void read_32(float* v, uint32_t from) {
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(from) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// Descriptor of an operand in shared memory: address, the two strides (in bytes) and the swizzle of 128 bytes.
__device__ __forceinline__ uint64_t operand(uint32_t address, uint32_t leading, uint32_t stride) {
    return (uint64_t)((address & 0x3FFFF) >> 4) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

struct Tile { uint32_t which, i, j; };                           // matrix, block of 128 rows, block of 256 columns

// Tiles on and below the diagonal: rows 2q and 2q + 1 have q + 1 tiles each, the rows before them q (q + 1).
__device__ __forceinline__ Tile gram_tile(const uint32_t* first, uint32_t n, uint32_t u) {
    Tile t;
    t.which = matrix_of(first, n, u);
    const uint32_t r = u - __ldg(first + t.which);
    uint32_t q = (uint32_t)((sqrtf(4.f * (float)r + 1.f) - 1.f) * 0.5f);
    while (q * (q + 1) > r) --q;
    while ((q + 1) * (q + 2) <= r) ++q;
    const uint32_t rest = r - q * (q + 1), second = rest >= q + 1;
    t.i = 2 * q + second;
    t.j = rest - second * (q + 1);
    return t;
}
// All tiles, a column's one after the other: they share the right operand.
__device__ __forceinline__ Tile apply_tile(const uint32_t* first, uint32_t n, uint32_t u, const PlanEntry* e) {
    Tile t;
    t.which = matrix_of(first, n, u);
    const uint32_t r = u - __ldg(first + t.which), mb = e[t.which].mb;
    t.j = r / mb;
    t.i = r - t.j * mb;
    return t;
}

__device__ __forceinline__ void pack8(unsigned char* to, const float* v) {       // 8 numbers (times 2^14) as float16
    uint4 r;
    uint32_t* w = &r.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) { const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
    *reinterpret_cast<uint4*>(to) = r;
}
__device__ __forceinline__ void unpack8(float* v, const unsigned char* from, bool more) {
    const uint4 r = *reinterpret_cast<const uint4*>(from);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = more ? v[2 * i] + f.x : f.x; v[2 * i + 1] = more ? v[2 * i + 1] + f.y : f.y;
    }
}
// 32 columns of a row in a block, from piece c on; what float16 leaves over goes to `low`.
__device__ __forceinline__ void put_32(unsigned char* block, unsigned char* low, uint32_t r, uint32_t c, float* v) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        pack8(block + piece(r, c + q), v + 8 * q);
        if (low) {
            float rest[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) rest[i] = v[8 * q + i] - __half2float(__float2half_rn(v[8 * q + i]));
            pack8(low + piece(r, c + q), rest);
        }
    }
}
__device__ __forceinline__ void get_32(float* v, const unsigned char* block, const unsigned char* low, uint32_t r, uint32_t c) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        unpack8(v + 8 * q, block + piece(r, c + q), false);
        if (low) unpack8(v + 8 * q, low + piece(r, c + q), true);
    }
}

// The sums of a tile's row in 32 columns, as entries of A, B or X, or the weights that they move.
template <int MODE> __device__ __forceinline__ void finish(const MuonArgs& a, const PlanEntry& t, uint32_t which, uint32_t bi, uint32_t r, uint32_t j0, float* v,
                                                           const unsigned char* x_in, unsigned char* x_out, float* stage) {
    const uint32_t i = bi * 128 + r, lane = threadIdx.x % 32;
    if (MODE == kGram || MODE == kPoly) {
        const uint32_t jb = j0 / 128;                            // block of 128 columns; above the diagonal: the other tile's
        if (jb > bi) return;
        const uint64_t here = (t.a_block + (uint64_t)bi * 2 * t.mb + j0 / 64) * kBlockBytes;
        unsigned char* out = (MODE == kGram ? a.a : a.b) + here;
        if (MODE == kGram) {
#pragma unroll
            for (int q = 0; q < 32; ++q) {
                if (j0 + q == i) { a.diag_a[t.diagonal + i] = v[q] * kDown2; v[q] = 0.f; }
                v[q] *= kDown;
            }
        } else {
            float e[32];
            get_32(e, a.a + here, a.split ? a.a + a.a_bytes + here : nullptr, r, j0 % 64 / 8);
            const float* d = a.diag_a + t.diagonal;
            const float di = d[i];
#pragma unroll
            for (int q = 0; q < 32; ++q) {
                const float dj = d[j0 + q];
                if (j0 + q == i) {
                    a.diag_b[t.diagonal + i] = fmaf(kQ5, fmaf(v[q], kDown2, di * di), kQ3 * di);
                    v[q] = 0.f;
                } else {
                    v[q] = fmaf(kQ5 * kDown, v[q], e[q] * fmaf(kQ5, di + dj, kQ3));
                }
            }
        }
        put_32(out, a.split ? out + a.a_bytes : nullptr, r, j0 % 64 / 8, v);
        if (jb == bi) return;
        // the same below: element (j, i), neighbours along i in neighbouring lanes
        unsigned char* mirror = (MODE == kGram ? a.a : a.b) + (t.a_block + (uint64_t)jb * 2 * t.mb + i / 64) * kBlockBytes;
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            const uint32_t row = (j0 + q) % 128, to = piece(row, i % 64 / 8) + i % 8 * 2;
            const __half h = __float2half_rn(v[q]);
            *reinterpret_cast<__half*>(mirror + to) = h;
            if (a.split) *reinterpret_cast<__half*>(mirror + a.a_bytes + to) = __float2half_rn(v[q] - __half2float(h));
        }
        return;
    }
    const uint64_t here = (t.x_block + (uint64_t)bi * t.nb + j0 / 64) * kBlockBytes;
    float e[32];
    get_32(e, x_in + here, a.split ? x_in + a.x_bytes + here : nullptr, r, j0 % 64 / 8);
    const float keep = kQ1 + a.diag_b[t.diagonal + i];
#pragma unroll
    for (int q = 0; q < 32; ++q) v[q] = fmaf(v[q], kDown, keep * e[q]);          // times 2^14
    if (MODE == kApply) {
        put_32(x_out + here, a.split ? x_out + a.x_bytes + here : nullptr, r, j0 % 64 / 8, v);
        return;
    }
    const float l = a.lr * t.lr_scale, down = 1.f - l * t.weight_decay, move = -l * kDown;
    void* const weights = t.master ? static_cast<void*>(t.master) : t.param;
    const uint32_t dtype = t.master ? FTC_F32 : t.param_dtype;
    if (!t.tall) {                                               // lanes have rows: turned, so that they have neighbouring columns
#pragma unroll
        for (int q = 0; q < 32; ++q) stage[lane * 33 + q] = v[q];
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 32; ++q) v[q] = stage[q * 33 + lane];
        __syncwarp();
    }
    const uint32_t i0 = i - lane;
#pragma unroll 8
    for (int q = 0; q < 32; ++q) {
        const uint32_t row = t.tall ? j0 + q : i0 + q, col = t.tall ? i : j0 + lane;
        if (row < t.rows && col < t.cols) {
            const uint64_t at = (uint64_t)row * t.cols + col;
            const float p = fmaf(element(weights, dtype, at), down, v[q] * move);
            set_element(weights, dtype, at, p);
            if (t.master) set_element(t.param, t.param_dtype, at, p);
        }
    }
}

template <int MODE> __global__ void __launch_bounds__(kProductThreads, 1) muon_product_kernel(MuonArgs a, uint32_t tiles, uint32_t side) {
    extern __shared__ unsigned char raw[];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    unsigned char* const smem = raw + (1024 - (smem_of(raw) & 1023)) % 1024;
    float* const stage_out = reinterpret_cast<float*>(smem + kStages * kStageBytes);
    uint64_t* const bars = reinterpret_cast<uint64_t*>(smem + kStages * kStageBytes + kOutBytes);    // full, empty, sums full, sums empty, drained
    uint32_t* const words = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 5);                     // tensor memory, gave up
    const uint32_t full = smem_of(bars), empty = full + 8 * kStages, sum_full = empty + 8 * kStages, sum_empty = sum_full + 16, drained = sum_empty + 16;
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kStages; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 1); }
        for (uint32_t s = 0; s < 2; ++s) { bar_init(sum_full + 8 * s, 1); bar_init(sum_empty + 8 * s, 4); }
        bar_init(drained, 1);
        words[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_of(words)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = words[0];
    wait_for_earlier_kernel();
    later_kernel_may_start();
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    const bool work = isfinite(scale) && *reinterpret_cast<volatile uint32_t*>(a.word) == 0;
    const PlanEntry* const entries = plan_entries(a.plan);
    const uint32_t* const first = plan_first(a.plan, a.n, MODE <= kPoly ? kGramFirst : kApplyFirst);
    const uint32_t segments = a.split ? 3 : 1;
    auto tile_of = [&](uint32_t u) { return MODE <= kPoly ? gram_tile(first, a.n, u) : apply_tile(first, a.n, u, entries); };
    const unsigned char* const x_in = a.x[side];
    bool ok = true;

    if (work && warp == 0 && lane == 0) {                        // copies
        uint32_t it = 0;
        for (uint32_t u = blockIdx.x; u < tiles && ok; u += gridDim.x) {
            const Tile tile = tile_of(u);
            const PlanEntry& t = entries[tile.which];
            const uint32_t steps = MODE == kGram ? t.nb : t.kb;
            const uint32_t right = MODE <= kPoly ? min(2u, t.mb - 2 * tile.j) : min(4u, t.nb - 4 * tile.j);
            const uint32_t bytes = kBlockBytes + right * (MODE <= kPoly ? kBlockBytes : kBlockBytes / 2);
            for (uint32_t g = 0; g < segments && ok; ++g) {
                const unsigned char* l = (MODE == kGram ? x_in : MODE == kPoly ? a.a : a.b) + (g == 2 ? (MODE == kGram ? a.x_bytes : a.a_bytes) : 0);
                const unsigned char* r = (MODE == kPoly ? a.a : x_in) + (g == 1 ? (MODE == kPoly ? a.a_bytes : a.x_bytes) : 0);
                for (uint32_t s = 0; s < steps; ++s, ++it) {
                    const uint32_t slot = it % kStages, to = smem_of(smem) + slot * kStageBytes, bar = full + 8 * slot;
                    if (it >= kStages && !(ok = bar_wait(empty + 8 * slot, (it / kStages - 1) & 1))) break;
                    bar_expect(bar, bytes);
                    if (MODE == kGram) {
                        copy_in(to, l + (t.x_block + (uint64_t)tile.i * t.nb + s) * kBlockBytes, kBlockBytes, bar);
                        for (uint32_t q = 0; q < right; ++q)
                            copy_in(to + (1 + q) * kBlockBytes, r + (t.x_block + (uint64_t)(2 * tile.j + q) * t.nb + s) * kBlockBytes, kBlockBytes, bar);
                    } else {
                        copy_in(to, l + (t.a_block + (uint64_t)tile.i * 2 * t.mb + s) * kBlockBytes, kBlockBytes, bar);
                        if (MODE == kPoly)
                            for (uint32_t q = 0; q < right; ++q)
                                copy_in(to + (1 + q) * kBlockBytes, r + (t.a_block + (uint64_t)(2 * tile.j + q) * 2 * t.mb + s) * kBlockBytes, kBlockBytes, bar);
                        else                                     // 64 rows of X (half a block), up to four blocks of 64 columns
                            for (uint32_t q = 0; q < right; ++q)
                                copy_in(to + kBlockBytes + q * (kBlockBytes / 2),
                                        r + (t.x_block + (uint64_t)(s / 2) * t.nb + 4 * tile.j + q) * kBlockBytes + s % 2 * (kBlockBytes / 2), kBlockBytes / 2, bar);
                    }
                }
            }
        }
        if (!ok) {                                               // copies in flight end before the block does
            words[1] = 1;
            for (uint32_t s = 0; s < kStages && s < it; ++s) bar_wait(full + 8 * s, ((it - 1 - s) / kStages) & 1);
        }
    } else if (work && warp == 1 && lane == 0) {                 // matrix instructions
        uint32_t it = 0, n = 0;
        for (uint32_t u = blockIdx.x; u < tiles && ok; u += gridDim.x, ++n) {
            const Tile tile = tile_of(u);
            const PlanEntry& t = entries[tile.which];
            const uint32_t steps = segments * (MODE == kGram ? t.nb : t.kb);
            const uint32_t columns = MODE <= kPoly ? min(2u, t.mb - 2 * tile.j) * 128 : min(4u, t.nb - 4 * tile.j) * 64;
            // sums in float32, operands float16, the right one along its columns in the apply kernels
            const uint32_t how = 1u << 4 | (MODE >= kApply ? 1u << 16 : 0u) | columns / 8 << 17 | 128u / 16 << 24;
            const uint32_t sum = tmem + (n & 1) * 256;
            if (n >= 2 && !(ok = bar_wait(sum_empty + 8 * (n & 1), (n / 2 - 1) & 1))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (uint32_t s = 0; s < steps; ++s, ++it) {
                const uint32_t slot = it % kStages, at = smem_of(smem) + slot * kStageBytes;
                if (!(ok = bar_wait(full + 8 * slot, (it / kStages) & 1))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {               // 16 of the inner dimension: 32 bytes along a row, 16 rows of 128 bytes
                    const uint64_t l = operand(at + k * 32, 16, 1024);
                    const uint64_t r = MODE <= kPoly ? operand(at + kBlockBytes + k * 32, 16, 1024) : operand(at + kBlockBytes + k * 2048, kBlockBytes / 2, 1024);
                    multiply(sum, l, r, how, s || k);
                }
                commit_to(empty + 8 * slot);
            }
            if (ok) commit_to(sum_full + 8 * (n & 1));
        }
        if (!ok) {
            words[1] = 1;
            commit_to(drained);                                  // products in flight end before the tensor memory is given back
            bar_wait(drained, 0);
        }
    } else if (work && warp >= 4) {                              // sums
        const uint32_t quarter = warp - 4, r = quarter * 32 + lane;
        uint32_t n = 0;
        for (uint32_t u = blockIdx.x; u < tiles; u += gridDim.x, ++n) {
            const Tile tile = tile_of(u);
            const PlanEntry& t = entries[tile.which];
            ok = __all_sync(0xFFFFFFFFu, bar_wait(sum_full + 8 * (n & 1), (n / 2) & 1));
            if (!ok) { if (lane == 0) words[1] = 1; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t columns = MODE <= kPoly ? min(2u, t.mb - 2 * tile.j) * 128 : min(4u, t.nb - 4 * tile.j) * 64;
            const bool wanted = MODE != kUpdate || a.live[tile.which];
            for (uint32_t c = 0; c < columns && wanted; c += 32) {
                float v[32];
                read_32(v, tmem + (n & 1) * 256 + (quarter * 32 << 16) + c);
                finish<MODE>(a, t, tile.which, tile.i, r, tile.j * 256 + c, v, x_in, a.x[side ^ 1], stage_out + quarter * 32 * 33);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(sum_empty + 8 * (n & 1));
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(words + 1)) *a.word = 1;
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <int MODE> static cudaError_t product(const MuonArgs& a, uint32_t tiles, uint32_t side, int sms, cudaStream_t st) {
    cudaError_t e = cudaFuncSetAttribute(muon_product_kernel<MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3(tiles < (uint32_t)sms ? tiles : (uint32_t)sms); how.blockDim = dim3(kProductThreads); how.dynamicSmemBytes = kProductSmem;
    how.stream = st; how.attrs = &early; how.numAttrs = 1;
    return cudaLaunchKernelEx(&how, muon_product_kernel<MODE>, a, tiles, side);
}

cudaError_t launch_muon(const MuonArgs& a, int sms, cudaStream_t st) {
    muon_momentum_kernel<<<a.chunks, 256, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_second(muon_layout_kernel, a.x_blocks, 256, st, a);
    for (uint32_t s = 0; s < a.steps && e == cudaSuccess; ++s) {
        e = product<kGram>(a, a.gram_tiles, s & 1, sms, st);
        if (e == cudaSuccess) e = product<kPoly>(a, a.gram_tiles, s & 1, sms, st);
        if (e == cudaSuccess) e = s + 1 < a.steps ? product<kApply>(a, a.apply_tiles, s & 1, sms, st) : product<kUpdate>(a, a.apply_tiles, s & 1, sms, st);
    }
    return e;
}

}  // namespace ftc
