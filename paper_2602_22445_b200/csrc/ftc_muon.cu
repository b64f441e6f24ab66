// Orthogonalised updates of many matrices: momentum, then Newton-Schulz steps X <- a X + (b A + c A A) X with A = X X^T, then the weights.
//
// Two kernels take the momentum and lay out X = U / |U| (m x w, m <= w: matrices with more rows than columns transposed), three products a
// step follow, each over all matrices at once:
//   gram   A = X X^T             symmetric: tiles on and below the diagonal, written twice
//   poly   B = b A + c A A       symmetric too (A A = A A^T)
//   apply  X = (a + B) X
// Operands are float16, held times 2^14: |X| stays below 1.21 after the first step (the largest value of the quintic on 0 .. 1.21), entries of
// A below 1.47 and of B below 2.81, so nothing overflows and numbers down to 2^-28 keep their 11 bits (bfloat16 would keep 8). Diagonals,
// which are the large entries of A and B in late steps, are held apart in float32: with A = D + A', A A = A' A' + D A' + A' D + D D, all but
// the first by elements; with B = E + B', X = B' X + (a + E) X, the second by elements too (E rounded with the rest: an error larger by 1.35 to 1.9).
// Sums are float32 throughout, in tensor memory.
// With `split` every operand is two float16 numbers, the second one what the first leaves over: hi lo + lo hi + hi hi in one sum, in this order: the
// tensor cores cut the sum to float32 every 16 products, of which the small ones' cuts count nothing while the large ones are not in it yet
// (hi hi first: 1.3 to 4 times the error). a + E, up to 3.45, is B's diagonal then (22 bits of it, as of all else).
//
// Matrices lie in the workspace in blocks of 128 rows x 64 columns (16 KB), their 16-byte pieces in the order that the tensor cores read
// (piece c of row r at c ^ r % 8): a block is one contiguous copy, whichever way a product reads it, and edges are zeros.
#include <cooperative_groups.h>
#include "ftc_f32x2.cuh"
#include "ftc_lm.cuh"

namespace ftc {

constexpr float kQ1 = 3.4445f, kQ3 = -4.7750f, kQ5 = 2.0315f;
constexpr float kUp = 16384.f, kDown = 1.f / 16384.f, kDown2 = kDown * kDown;    // 2^14
constexpr uint32_t kBlockBytes = 128 * 64 * 2;

// What the gradient is multiplied with: 1 / processes included, 0: not delivered.
__device__ __forceinline__ float share_at(const PlanEntry& t, uint64_t i) {
    if (!t.status) return 1.f;
    const uint64_t q = t.k_shift != 255 ? i >> t.k_shift : (uint32_t)i / t.k;
    const uint2 s = *reinterpret_cast<const uint2*>(t.status + q * FTC_STATUS_WORDS);
    return (s.x & 0xFFu) == FTC_ST_OK && s.y ? 1.f / (float)s.y : 0.f;
}

// N elements at at(0), at(1), ... where there(i): all loads out before anything else.
template <typename T, int N, typename A, typename B> __device__ __forceinline__ void gather_of(float (&v)[N], const T* p, A at, B there) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = there(i) ? to_f32(p[at(i)]) : 0.f;
}
template <int N, typename A, typename B> __device__ __forceinline__ void gather(float (&v)[N], const void* p, uint32_t dtype, A at, B there) {
    if (dtype == FTC_F32) gather_of(v, static_cast<const float*>(p), at, there);
    else if (dtype == FTC_BF16) gather_of(v, static_cast<const __nv_bfloat16*>(p), at, there);
    else gather_of(v, static_cast<const __half*>(p), at, there);
}
template <typename T, int N, typename A, typename B> __device__ __forceinline__ void scatter_of(const float (&v)[N], T* p, A at, B there) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (there(i)) p[at(i)] = from_f32<T>(v[i]);
}
template <int N, typename A, typename B> __device__ __forceinline__ void scatter(const float (&v)[N], void* p, uint32_t dtype, A at, B there) {
    if (dtype == FTC_F32) scatter_of(v, static_cast<float*>(p), at, there);
    else if (dtype == FTC_BF16) scatter_of(v, static_cast<__nv_bfloat16*>(p), at, there);
    else scatter_of(v, static_cast<__half*>(p), at, there);
}
template <int N, typename A, typename B> __device__ __forceinline__ void gather_shares(float (&v)[N], const PlanEntry& t, A at, B there) {
    if (!t.status) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = there(i) ? 1.f : 0.f;
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = there(i) ? share_at(t, at(i)) : 0.f;
}

// ---- momentum ----

// Eight neighbouring elements as numbers.
__device__ __forceinline__ void eight(float* v, const void* p, uint32_t dtype, uint64_t i) {
    if (dtype == FTC_F32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
        const float4 a = q[0], b = q[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        return;
    }
    const uint4 r = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (dtype == FTC_BF16) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u); }
        else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j])); v[2 * j] = f.x; v[2 * j + 1] = f.y; }
    }
}
__device__ __forceinline__ void store_eight(void* p, uint32_t dtype, uint64_t i, const float* v) {
    if (dtype == FTC_F32) {
        float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
        q[0] = make_float4(v[0], v[1], v[2], v[3]); q[1] = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
    uint4 r;
    uint32_t* w = &r.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (dtype == FTC_BF16) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]); w[j] = *reinterpret_cast<const uint32_t*>(&h); }
        else { const __half2 h = __floats2half2_rn(v[2 * j], v[2 * j + 1]); w[j] = *reinterpret_cast<const uint32_t*>(&h); }
    }
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) = r;
}
// Shares of eight neighbours; messages of a multiple of 8 elements have one for all.
__device__ __forceinline__ void eight_shares(float* s, const PlanEntry& t, uint64_t i) {
    const float one = share_at(t, i);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = t.status && t.k % 8 ? share_at(t, i + j) : one;
}

// A block has 4096 elements of one matrix: twice eight a thread, neighbours where the addresses allow it (t.wide), 256 apart otherwise; all loads
// are out before the first is used (24 of 1024 x 1024 in float32, 302 MB: 50 us, 6.0 TB/s).
__global__ void __launch_bounds__(256, 4) muon_momentum_kernel(MuonArgs a) {
    later_kernel_may_start();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.word = 0;
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!isfinite(scale)) return;
    const uint32_t which = a.maps[kChunks][blockIdx.x];
    const PlanEntry t = plan_entries(a.plan)[which];
    const uint64_t begin = (uint64_t)(blockIdx.x - t.first[kChunks]) * kMuonChunk;
    const uint32_t left = (uint32_t)min((uint64_t)kMuonChunk, t.n - begin);
    float* m = a.momentum + t.first_block * FTC_STATE_BLOCK + begin;
    float old[16], g[16], s[16];
    const bool wide = t.wide && left == kMuonChunk;
    auto at = [&](int j) { return (uint32_t)(threadIdx.x + j * 256); };
    auto there = [&](int j) { return at(j) < left; };
    if (wide) {
#pragma unroll
        for (uint32_t w = 0; w < 2; ++w) {
            const uint32_t e = (w * 256 + threadIdx.x) * 8;
            eight(old + 8 * w, m, FTC_F32, e);
            eight(g + 8 * w, t.grad, t.grad_dtype, begin + e);
            eight_shares(s + 8 * w, t, begin + e);
        }
    } else {
        gather(old, m, FTC_F32, at, there);
        gather(g, t.grad, t.grad_dtype, [&](int j) { return begin + at(j); }, there);
        gather_shares(s, t, [&](int j) { return begin + at(j); }, there);
    }
    double sum = 0;
    uint32_t live = 0;
#pragma unroll
    for (uint32_t j = 0; j < 16; ++j) {
        float u = old[j];
        if (s[j] > 0.f) {
            const float d = g[j] * s[j] * scale;
            old[j] = fmaf(old[j], a.mu, d);
            u = a.nesterov ? fmaf(old[j], a.mu, d) : old[j];
            live |= 1u << j;
        }
        sum = ::fma((double)u, (double)u, sum);
    }
    if (wide) {
#pragma unroll
        for (uint32_t w = 0; w < 2; ++w)
            if (live >> (8 * w) & 0xFFu) store_eight(m, FTC_F32, (w * 256 + threadIdx.x) * 8, old + 8 * w);
    } else {
        scatter(old, m, FTC_F32, at, [&](int j) { return live >> j & 1u; });
    }
    __shared__ double sums[8];
    __shared__ uint32_t lives[8];
    sum = warp_sum(sum);
    live = __any_sync(0xFFFFFFFFu, live != 0);
    if (threadIdx.x % 32 == 0) { sums[threadIdx.x / 32] = sum; lives[threadIdx.x / 32] = live; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) { sum += sums[w]; live |= lives[w]; }
        a.sums[blockIdx.x] = make_double2(sum, live ? 1.0 : 0.0);
    }
}

// A matrix's factor 2^14 / (|U| + eps), and whether anything of it was delivered: its chunks' sums in a fixed order.
__global__ void __launch_bounds__(256) muon_norm_kernel(MuonArgs a) {
    wait_for_earlier_kernel();
    later_kernel_may_start();
    const PlanEntry& t = plan_entries(a.plan)[blockIdx.x];
    const uint32_t c0 = t.first[kChunks], c1 = c0 + (uint32_t)((t.n + kMuonChunk - 1) / kMuonChunk);
    __shared__ double sums[8], lives[8];
    double sum = 0, live = 0;
#pragma unroll 4
    for (uint32_t c = c0 + threadIdx.x; c < c1; c += 256) { const double2 s = a.sums[c]; sum += s.x; live += s.y; }
    sum = warp_sum(sum); live = warp_sum(live);
    if (threadIdx.x % 32 == 0) { sums[threadIdx.x / 32] = sum; lives[threadIdx.x / 32] = live; }
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 8; ++w) { sum += sums[w]; live += lives[w]; }
    a.live[blockIdx.x] = live > 0;
    for (uint32_t k = 0; k < 3; ++k) a.written[k * a.n + blockIdx.x] = 0;
    a.factor[blockIdx.x] = (float)((double)kUp / (sqrt(sum) + (double)a.eps));
}

// Where the 16-byte piece c of row r lies in a block.
__device__ __forceinline__ uint32_t piece(uint32_t r, uint32_t c) { return r * 128 + ((c ^ (r & 7)) << 4); }

// A transposed block is turned in shared memory as float32, 64 lines of 128 with a gap of 4 behind each and behind every eighth: whole lines are
// written and read by neighbouring threads in 16 bytes each, columns by neighbouring threads in neighbouring words or eight lines apart.
constexpr uint32_t kTurnBytes = (64 * 132 + 32) * 4;
__device__ __forceinline__ uint32_t turn_line(uint32_t line) { return line * 132 + line / 8 * 4; }
static_assert(kTurnBytes >= 2 * kBlockBytes, "a block's two numbers take the same memory");

// One block of 128 x 64 of X. Elements that are neighbours in memory are loaded by one thread (eight, where the addresses allow it) or by
// neighbouring threads; a block whose matrix is transposed is turned in shared memory (24 of 4096 x 1024: 233 us when threads took a line each, 160 so;
// of 1024 x 4096, nothing turned: 151). Bound by loads in flight: four blocks an SM, 64 registers a thread (three blocks: 10 % more, five: 10 % too).
__global__ void __launch_bounds__(256, 4) muon_layout_kernel(MuonArgs a) {
    wait_for_earlier_kernel();
    later_kernel_may_start();
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!isfinite(scale)) return;
    const uint32_t which = a.maps[kBlocks][blockIdx.x];
    const PlanEntry t = plan_entries(a.plan)[which];
    const uint32_t at = blockIdx.x - t.first[kBlocks], bi = at / t.nb, bj = at - bi * t.nb;
    const float inv = a.factor[which];
    const float* m = a.momentum + t.first_block * FTC_STATE_BLOCK;
    __shared__ __align__(16) unsigned char room[kTurnBytes];
    unsigned char* const out = a.x[0] + (t.x_block + at) * kBlockBytes;
    auto value = [&](float v, float g, float s) { return (a.nesterov && s > 0.f ? fmaf(v, a.mu, g * s * scale) : v) * inv; };
    auto put = [&](uint32_t r, uint32_t c, float v) {
        const __half h = __float2half_rn(v);
        const uint32_t to = piece(r, c / 8) + c % 8 * 2;
        *reinterpret_cast<__half*>(room + to) = h;
        if (a.split) *reinterpret_cast<__half*>(room + kBlockBytes + to) = __float2half_rn(v - __half2float(h));
    };
    auto put_eight = [&](unsigned char* to, uint64_t low, float* x) {
        store_eight(to, FTC_F16, 0, x);
        if (a.split) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] -= __half2float(__float2half_rn(x[j]));
            store_eight(to + low, FTC_F16, 0, x);
        }
    };
    if (bi * 128 + 128 <= t.m && bj * 64 + 64 <= t.w && t.wide && t.cols % 8 == 0) {
        // runs of 64 neighbours in 128 lines of memory, or of 128 in 64 (transposed)
        float* const turn = reinterpret_cast<float*>(room);
#pragma unroll
        for (uint32_t u = 0; u < 2; ++u) {
            float v[2][8], g[2][8], s[2][8];
            uint32_t line[2], run[2];
#pragma unroll
            for (uint32_t w = 0; w < 2; ++w) {
                const uint32_t e = threadIdx.x + (2 * u + w) * 256;
                line[w] = t.tall ? e / 16 : e / 8;
                run[w] = t.tall ? e % 16 * 8 : e % 8 * 8;
                const uint64_t q = t.tall ? (uint64_t)(bj * 64 + line[w]) * t.cols + bi * 128 + run[w] : (uint64_t)(bi * 128 + line[w]) * t.cols + bj * 64 + run[w];
                eight(v[w], m, FTC_F32, q);
                if (a.nesterov) { eight(g[w], t.grad, t.grad_dtype, q); eight_shares(s[w], t, q); }
            }
#pragma unroll
            for (uint32_t w = 0; w < 2; ++w) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = value(v[w][j], g[w][j], s[w][j]);
                if (t.tall) store_eight(turn + turn_line(line[w]) + run[w], FTC_F32, 0, x);
                else put_eight(out + piece(line[w], run[w] / 8), a.x_bytes, x);
            }
        }
        if (!t.tall) return;
        float x[4][8];
        const uint32_t r = threadIdx.x % 128, c0 = threadIdx.x / 128;
        __syncthreads();
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) x[u][j] = turn[turn_line((c0 + 2 * u) * 8 + j) + r];
        __syncthreads();
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) put_eight(room + piece(r, c0 + 2 * u), kBlockBytes, x[u]);
    } else {
        for (uint32_t e0 = threadIdx.x; e0 < 128 * 64; e0 += 2048) {
            float v[8], g[8] = {}, s[8] = {};
            auto row = [&](int w) { const uint32_t e = e0 + w * 256; return t.tall ? e % 128 : e / 64; };
            auto col = [&](int w) { const uint32_t e = e0 + w * 256; return t.tall ? e / 128 : e % 64; };
            auto there = [&](int w) { return bi * 128 + row(w) < t.m && bj * 64 + col(w) < t.w; };
            auto place = [&](int w) {
                const uint32_t i = bi * 128 + row(w), j = bj * 64 + col(w);
                return t.tall ? (uint64_t)j * t.cols + i : (uint64_t)i * t.cols + j;
            };
            gather(v, m, FTC_F32, place, there);
            if (a.nesterov) { gather(g, t.grad, t.grad_dtype, place, there); gather_shares(s, t, place, there); }
#pragma unroll
            for (int w = 0; w < 8; ++w) put(row(w), col(w), value(v[w], g[w], s[w]));
        }
    }
    __syncthreads();
    for (uint32_t s = 0; s <= a.split; ++s) {
        uint4* to = reinterpret_cast<uint4*>(out + s * a.x_bytes);
        const uint4* from = reinterpret_cast<const uint4*>(room + s * kBlockBytes);
        for (uint32_t e = threadIdx.x; e < kBlockBytes / 16; e += 256) to[e] = from[e];
    }
}

// The weights that one block of 128 x 64 of X moves; elements as in the layout (24 of 1024 x 4096 in float32: 176 us, 5.7 TB/s; of 4096 x 1024: 207).
__global__ void __launch_bounds__(256, 4) muon_update_kernel(MuonArgs a) {
    wait_for_earlier_kernel();
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    const uint32_t which = a.maps[kBlocks][blockIdx.x];
    if (!isfinite(scale) || *reinterpret_cast<volatile uint32_t*>(a.word) || !a.live[which]) return;
    const PlanEntry t = plan_entries(a.plan)[which];
    const uint32_t at = blockIdx.x - t.first[kBlocks], bi = at / t.nb, bj = at - bi * t.nb;
    const unsigned char* const x_at = a.x[a.steps & 1] + (t.x_block + at) * kBlockBytes;
    const float l = a.lr * t.lr_scale, down = 1.f - l * t.weight_decay, move = -l * kDown;
    void* const weights = t.master ? static_cast<void*>(t.master) : t.param;
    const uint32_t dtype = t.master ? FTC_F32 : t.param_dtype;
    __shared__ __align__(16) unsigned char room[kTurnBytes];
    const bool whole = bi * 128 + 128 <= t.m && bj * 64 + 64 <= t.w && t.wide && t.cols % 8 == 0;
    if (whole && !t.tall) {                                      // pieces as they are
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            float p[2][8], x[2][8], y[2][8];
            uint64_t place[2];
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {
                const uint32_t e = threadIdx.x + (2 * h + u) * 256, line = e / 8, run = e % 8 * 8;
                place[u] = (uint64_t)(bi * 128 + line) * t.cols + bj * 64 + run;
                eight(p[u], weights, dtype, place[u]);
                eight(x[u], x_at + piece(line, run / 8), FTC_F16, 0);
                if (a.split) eight(y[u], x_at + a.x_bytes + piece(line, run / 8), FTC_F16, 0);
            }
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) p[u][j] = fmaf(p[u][j], down, (a.split ? x[u][j] + y[u][j] : x[u][j]) * move);
                store_eight(weights, dtype, place[u], p[u]);
                if (t.master) store_eight(t.param, t.param_dtype, place[u], p[u]);
            }
        }
        return;
    }
    if (whole) {                                                 // turned
        float* const turn = reinterpret_cast<float*>(room);
        float p[4][8];
        const uint32_t line = threadIdx.x / 16, run = threadIdx.x % 16 * 8;      // and every 16th line after
        const uint64_t place = (uint64_t)(bj * 64 + line) * t.cols + bi * 128 + run, on = (uint64_t)16 * t.cols;
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) eight(p[u], weights, dtype, place + u * on);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t e = threadIdx.x + u * 256, r = e / 8, c = (e & 7) ^ (r & 7);      // a row's pieces as they lie: neighbours in memory
            float x[8], y[8];
            eight(x, x_at + e * 16, FTC_F16, 0);
            if (a.split) eight(y, x_at + a.x_bytes + e * 16, FTC_F16, 0);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) turn[turn_line(c * 8 + j) + r] = a.split ? x[j] + y[j] : x[j];
        }
        __syncthreads();
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            float x[8];
            eight(x, turn + turn_line(line + u * 16) + run, FTC_F32, 0);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) p[u][j] = fmaf(p[u][j], down, x[j] * move);
            store_eight(weights, dtype, place + u * on, p[u]);
            if (t.master) store_eight(t.param, t.param_dtype, place + u * on, p[u]);
        }
        return;
    }
    for (uint32_t s = 0; s <= a.split; ++s) {
        const uint4* from = reinterpret_cast<const uint4*>(x_at + s * a.x_bytes);
        uint4* to = reinterpret_cast<uint4*>(room + s * kBlockBytes);
#pragma unroll
        for (uint32_t e = 0; e < kBlockBytes / 16 / 256; ++e) to[threadIdx.x + e * 256] = from[threadIdx.x + e * 256];
    }
    auto update = [&](uint32_t r, uint32_t c) {
        const uint32_t q = piece(r, c / 8) + c % 8 * 2;
        float v = __half2float(*reinterpret_cast<const __half*>(room + q));
        if (a.split) v += __half2float(*reinterpret_cast<const __half*>(room + kBlockBytes + q));
        return v * move;
    };
    __syncthreads();
    for (uint32_t e0 = threadIdx.x; e0 < 128 * 64; e0 += 2048) {
        float v[8];
        auto row = [&](int w) { const uint32_t e = e0 + w * 256; return t.tall ? e % 128 : e / 64; };
        auto col = [&](int w) { const uint32_t e = e0 + w * 256; return t.tall ? e / 128 : e % 64; };
        auto there = [&](int w) { return bi * 128 + row(w) < t.m && bj * 64 + col(w) < t.w; };
        auto place = [&](int w) {
            const uint32_t i = bi * 128 + row(w), j = bj * 64 + col(w);
            return t.tall ? (uint64_t)j * t.cols + i : (uint64_t)i * t.cols + j;
        };
        gather(v, weights, dtype, place, there);
#pragma unroll
        for (int w = 0; w < 8; ++w) v[w] = fmaf(v[w], down, update(row(w), col(w)));
        scatter(v, weights, dtype, place, there);
        if (t.master) scatter(v, t.param, t.param_dtype, place, there);
    }
}

// ---- products ----
//
// Persistent pairs of blocks (clusters of two), 12 warps each. A pair has a tile of 256 x 256: a block holds 128 rows of the left operand and
// half of the right one's columns, one thread of the first block issues the matrix instructions of both, and each block's tensor memory
// gets its 128 rows of sums, 256 columns; there are two such halves, so that one tile is read out while the next is multiplied. A stage
// holds 64 of the inner dimension: 16 KB of each operand in each block.
// All products of all steps are one launch. A pair takes every so many-th tile of their list; a tile waits until the product before it of its own
// matrix has been written, which with many matrices it long has been: no product's last tiles keep the GPU waiting, and none pays for a launch.
//   warp 0   copies of its block's operands
//   warp 1   first block: matrix instructions; second block: tells the first when its copies have landed
//   warps 4 .. 11   read sums out (a warp reads the 32 lanes of tensor memory that its number modulo 4 gives it), the first four those of the
//            left 128 columns, the others the right ones', 64 at a time, each warp for itself: what the result needs of A or X comes into shared
//            memory as 4 KB, is replaced there by the result, and goes out as 4 KB; its transpose in stores of 64 bytes.
// A step of 64 takes 0.47 us a pair (4096 x 4096), where the tensor cores alone would take 0.3: copies out of L2 bound it. 0.54 with 24 of
// 1024 x 4096 (five steps: 1.6 ms, 1.05 PFLOP/s with symmetric products counted half), where a tile's beginning and end count; finding the next tile
// while one is at work cost more than it gave (1.64 ms).

constexpr uint32_t kStages = 5, kStageBytes = 2 * kBlockBytes, kRows = kBlockBytes / 4, kProductThreads = 384;
constexpr uint32_t kProductSmem = kStages * kStageBytes + 16 * kRows + 1024 + 512;
static_assert(kProductSmem <= 227 * 1024, "shared memory of a block");
enum { kGram, kPoly, kApply };
template <int M> struct Mode { static constexpr int value = M; };

__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrives at the barrier of the pair's block `rank`.
__device__ __forceinline__ void bar_arrive_at(uint32_t bar, uint32_t rank) {
    asm volatile("{\n\t.reg .b32 there;\n\tmapa.shared::cluster.u32 there, %0, %1;\n\tmbarrier.arrive.shared::cluster.b64 _, [there];\n\t}"
                 ::"r"(bar), "r"(rank) : "memory");
}
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
__device__ __forceinline__ void copy_out(void* to, uint32_t from, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
}
// The barriers of both blocks of a pair get to know when all products issued so far are done.
__device__ __forceinline__ void commit_to_both(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t how, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
// 64 columns of a lane.
__device__ __forceinline__ void read_64(F2* v, uint32_t from) {
    uint32_t r[64];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(from + 0) : "memory");
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
                 : "r"(from + 32) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = pair(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
}

// Descriptor of an operand in shared memory: address, the two strides (in bytes) and the swizzle of 128 bytes.
__device__ __forceinline__ uint64_t operand(uint32_t address, uint32_t leading, uint32_t stride) {
    return (uint64_t)((address & 0x3FFFF) >> 4) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

struct Tile { uint32_t step, mode, which, i, j; };               // step, product, matrix, blocks of 256 rows and of 256 columns

// Tile u of a call: step by step, gram, poly and apply of all matrices; of a symmetric product the tiles on and below the diagonal (row i has i + 1), of
// the others a column's tiles one after the other: they share the right operand.
__device__ __forceinline__ Tile tile_at(const MuonArgs& a, uint32_t u) {
    Tile t;
    const uint32_t gram = a.items[kGramTiles], all = 2 * gram + a.items[kApplyTiles];
    t.step = u / all;
    uint32_t r = u - t.step * all;
    t.mode = r < gram ? kGram : r < 2 * gram ? kPoly : kApply;
    if (t.mode == kApply) {
        r -= 2 * gram;
        t.which = __ldg(a.maps[kApplyTiles] + r);
        const PlanEntry& e = plan_entries(a.plan)[t.which];
        const uint32_t rows = (e.mb + 1) / 2;
        r -= e.first[kApplyTiles];
        t.j = r / rows;
        t.i = r - t.j * rows;
        return t;
    }
    if (t.mode == kPoly) r -= gram;
    t.which = __ldg(a.maps[kGramTiles] + r);
    r -= plan_entries(a.plan)[t.which].first[kGramTiles];
    uint32_t i = (uint32_t)((sqrtf(8.f * (float)r + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1) / 2 > r) --i;
    while ((i + 1) * (i + 2) / 2 <= r) ++i;
    t.i = i;
    t.j = r - i * (i + 1) / 2;
    return t;
}

// What a tile reads is there once all tiles of its matrix's product before have been written: 16 warps count each of them.
__device__ __forceinline__ bool wait_for_product(const MuonArgs& a, const Tile& q, const PlanEntry& t) {
    const uint32_t rows = (t.mb + 1) / 2, gram = rows * (rows + 1) / 2, apply = rows * ((t.nb + 3) / 4);
    const uint32_t target = q.mode == kGram ? q.step * apply * 16 : (q.step + 1) * gram * 16;
    const uint32_t* const count = a.written + (q.mode == kGram ? 2 : q.mode - 1) * a.n + q.which;
    for (uint32_t i = 0; i < 1u << 23; ++i) {
        uint32_t now;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(now) : "l"(count) : "memory");
        if (now >= target) {
            asm volatile("fence.proxy.async;" ::: "memory");     // and for the copies that follow
            return true;
        }
        __nanosleep(64);
    }
    return false;
}

__device__ __forceinline__ uint32_t half2_of(F2 v) { uint32_t r; asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi(v)), "f"(lo(v))); return r; }
__device__ __forceinline__ F2 pair_of(uint32_t h) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h)); return pair(f.x, f.y); }

template <bool SPLIT> __global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1) muon_products_kernel(MuonArgs a) {
    namespace cg = cooperative_groups;
    extern __shared__ unsigned char raw[];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    unsigned char* const smem = raw + (1024 - (smem_of(raw) & 1023)) % 1024;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(smem + kStages * kStageBytes + 16 * kRows);
    // full, landed in the second block, empty (each stage); sums full, sums empty (two each); drained; warps' rows (two each)
    const uint32_t full = smem_of(bars), landed = full + 8 * kStages, empty = landed + 8 * kStages, sum_full = empty + 8 * kStages, sum_empty = sum_full + 16,
                   drained = sum_empty + 16, warp_full = drained + 8;
    uint32_t* const words = reinterpret_cast<uint32_t*>(bars + 3 * kStages + 21);                    // tensor memory, gave up
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kStages; ++s) { bar_init(full + 8 * s, 1); bar_init(landed + 8 * s, 1); bar_init(empty + 8 * s, 1); }
        for (uint32_t s = 0; s < 2; ++s) { bar_init(sum_full + 8 * s, 1); bar_init(sum_empty + 8 * s, 16); }
        for (uint32_t s = 0; s < 16; ++s) bar_init(warp_full + 8 * s, 1);
        bar_init(drained, 1);
        words[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_of(words)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cg::this_cluster().sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = words[0], pairs = gridDim.x / 2, our_pair = blockIdx.x / 2;
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    const bool work = isfinite(scale);                           // not by the word: another pair may be setting it, and threads would disagree
    const PlanEntry* const entries = plan_entries(a.plan);
    const uint32_t tiles = a.steps * (2 * a.items[kGramTiles] + a.items[kApplyTiles]);
    constexpr uint32_t segments = SPLIT ? 3 : 1;
    // a tile on the diagonal: the left operand is the right one too (hi hi, the last segment)
    auto one_of = [&](const PlanEntry& t, const Tile& q, uint32_t g) { return q.mode <= kPoly && g + 1 == segments && q.i == q.j && t.mb > 2 * q.j + 1; };
    auto inner_of = [&](const PlanEntry& t, const Tile& q) { return q.mode == kGram ? t.nb : t.kb; };             // blocks of 64
    // a tile's columns: 256, or 128 where there are no more (of an apply tile up to 64 of them are nobody's)
    auto columns_of = [&](const PlanEntry& t, const Tile& q) { return (q.mode <= kPoly ? t.mb > 2 * q.j + 1 : t.nb > 4 * q.j + 2) ? 256u : 128u; };
    bool ok = true;

    if (work && warp == 0 && lane == 0) {                        // copies
        uint32_t it = 0;
        for (uint32_t u = our_pair; u < tiles && ok; u += pairs) {
            const Tile tile = tile_at(a, u);
            const PlanEntry t = entries[tile.which];
            if (!(ok = wait_for_product(a, tile, t))) break;
            const bool sym = tile.mode <= kPoly, gram = tile.mode == kGram;
            const unsigned char* const x_in = a.x[tile.step & 1];
            const uint32_t steps = inner_of(t, tile), left_row = 2 * tile.i + rank, half = columns_of(t, tile) / 2;      // columns of this block
            const bool has_left = left_row < t.mb;
            // right operand of a symmetric product: rows half * rank .. of 256; of the others: blocks of 64 columns
            const uint32_t right_row = 2 * tile.j + (half == 128 ? rank : 0), right_in = half == 128 ? 0 : rank * (kBlockBytes / 2);
            const uint32_t right_block = 4 * tile.j + rank * (half / 64), right_blocks = sym ? 0 : min(half / 64, t.nb > right_block ? t.nb - right_block : 0u);
            for (uint32_t g = 0; g < segments && ok; ++g) {
                const bool one = one_of(t, tile, g);
                const uint32_t bytes = (has_left ? kBlockBytes : 0) + (one ? 0 : sym ? half * 128 : right_blocks * (kBlockBytes / 2));
                const unsigned char* l = (gram ? x_in : (tile.mode == kPoly) ? a.a : a.b) + (SPLIT && g == 1 ? (gram ? a.x_bytes : a.a_bytes) : 0);
                const unsigned char* r = ((tile.mode == kPoly) ? a.a : x_in) + (SPLIT && g == 0 ? ((tile.mode == kPoly) ? a.a_bytes : a.x_bytes) : 0);
                l += gram ? (t.x_block + (uint64_t)left_row * t.nb) * kBlockBytes : (t.a_block + (uint64_t)left_row * 2 * t.mb) * kBlockBytes;
                r += gram ? (t.x_block + (uint64_t)right_row * t.nb) * kBlockBytes + right_in
                   : (tile.mode == kPoly) ? (t.a_block + (uint64_t)right_row * 2 * t.mb) * kBlockBytes + right_in : (t.x_block + right_block) * kBlockBytes;
                for (uint32_t s = 0; s < steps; ++s, ++it) {
                    const uint32_t slot = it % kStages, to = smem_of(smem) + slot * kStageBytes, bar = full + 8 * slot;
                    if (it >= kStages && !(ok = bar_wait(empty + 8 * slot, (it / kStages - 1) & 1))) break;
                    bar_expect(bar, bytes);
                    if (has_left) copy_in(to, l + (uint64_t)s * kBlockBytes, kBlockBytes, bar);
                    if (one) continue;
                    if (sym) copy_in(to + kBlockBytes, r + (uint64_t)s * kBlockBytes, half * 128, bar);
                    else                                         // 64 rows of X (half a block)
                        for (uint32_t q = 0; q < right_blocks; ++q)
                            copy_in(to + kBlockBytes + q * (kBlockBytes / 2), r + ((uint64_t)(s / 2) * t.nb + q) * kBlockBytes + s % 2 * (kBlockBytes / 2), kBlockBytes / 2, bar);
                }
            }
        }
        if (!ok) {                                               // copies in flight end before the block does
            words[1] = 1;
            for (uint32_t s = 0; s < kStages && s < it; ++s) { const uint32_t n = it - 1 - s; bar_wait(full + 8 * (n % kStages), (n / kStages) & 1); }
        }
    } else if (work && warp == 1 && lane == 0) {
        uint32_t it = 0, n = 0;
        for (uint32_t u = our_pair; u < tiles && ok; u += pairs, ++n) {
            const Tile tile = tile_at(a, u);
            const PlanEntry t = entries[tile.which];
            const uint32_t inner = inner_of(t, tile), steps = segments * inner;
            if (rank) {                                          // the second block's copies
                for (uint32_t s = 0; s < steps; ++s, ++it) {
                    const uint32_t slot = it % kStages;
                    if (!(ok = bar_wait(full + 8 * slot, (it / kStages) & 1))) break;
                    bar_arrive_at(landed + 8 * slot, 0);
                }
                continue;
            }
            const bool sym = tile.mode <= kPoly;
            const uint32_t along = sym ? 32 : 2048, leading = sym ? 16 : kBlockBytes / 2;
            // sums in float32, operands float16, the right one along its columns in the apply kernels, 256 rows
            const uint32_t how = 1u << 4 | (!sym ? 1u << 16 : 0u) | columns_of(t, tile) / 8 << 17 | 256u / 16 << 24;
            const uint32_t sum = tmem + (n & 1) * 256;
            if (n >= 2 && !(ok = bar_wait(sum_empty + 8 * (n & 1), (n / 2 - 1) & 1))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (uint32_t s = 0; s < steps; ++s, ++it) {
                const uint32_t slot = it % kStages, at = smem_of(smem) + slot * kStageBytes;
                if (!(ok = bar_wait(full + 8 * slot, (it / kStages) & 1) && bar_wait(landed + 8 * slot, (it / kStages) & 1))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t right = at + (one_of(t, tile, s < (segments - 1) * inner ? 0 : segments - 1) ? 0 : kBlockBytes);
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {               // 16 of the inner dimension: 32 bytes along a row, 16 rows of 128 bytes
                    const uint64_t l = operand(at + k * 32, 16, 1024), r = operand(right + k * along, leading, 1024);
                    multiply(sum, l, r, how, s || k);
                }
                commit_to_both(empty + 8 * slot);
            }
            if (ok) commit_to_both(sum_full + 8 * (n & 1));
        }
        if (!ok) {
            words[1] = 1;
            if (!rank) {                                         // products in flight end before the tensor memory is given back
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(drained) : "memory");
                bar_wait(drained, 0);
            }
        }
    } else if (work && warp >= 4) {                              // sums
        const uint32_t team = (warp - 4) / 4, quarter = warp & 3, r = quarter * 32 + lane;
        // a warp's 32 rows of a block of 64 columns (4 KB, the block's rows in order); the low numbers, or the rows of the next 64 columns
        unsigned char* const mine = smem + kStages * kStageBytes + (warp - 4) * 2 * kRows;
        unsigned char* const other = mine + kRows;
        const uint32_t ready = warp_full + 16 * (warp - 4);
        uint32_t n = 0, done[2] = {0, 0};                        // phases of the two barriers
        // One tile's part of this warp, for each of the three products.
        auto finish = [&](auto mode, const Tile& tile, const PlanEntry& t) {
            constexpr int MODE = decltype(mode)::value;
            constexpr bool NEEDS = MODE == kPoly || (MODE == kApply && !SPLIT);          // what a diagonal multiplies: A, or X itself
            const uint32_t bi = 2 * tile.i + rank, i = bi * 128 + r;
            // blocks of 64 columns of this team: none above the diagonal, none beyond the edges
            const uint32_t cb0 = 4 * tile.j + 2 * team, edge = MODE <= kPoly ? 2 * min(t.mb, bi + 1) : t.nb;
            const uint32_t wanted = bi < t.mb && cb0 < edge ? min(2u, edge - cb0) : 0;
            const uint64_t row_at = (MODE <= kPoly ? t.a_block + (uint64_t)bi * 2 * t.mb : t.x_block + (uint64_t)bi * t.nb) * kBlockBytes + quarter * kRows;
            unsigned char* const out = (MODE == kGram ? a.a : MODE == kPoly ? a.b : a.x[tile.step & 1 ^ 1]) + row_at;
            const uint64_t low = MODE <= kPoly ? a.a_bytes : a.x_bytes;
            auto fetch = [&](uint32_t b, unsigned char* to, uint32_t bar) {              // by one lane
                const unsigned char* from = (MODE == kPoly ? a.a : a.x[tile.step & 1]) + row_at + (uint64_t)(cb0 + b) * kBlockBytes;
                bar_expect(bar, (SPLIT ? 2 : 1) * kRows);
                copy_in(smem_of(to), from, kRows, bar);
                if (SPLIT) copy_in(smem_of(other), from + low, kRows, bar);
            };
            if (NEEDS && wanted && lane == 0) ok = wait_for_product(a, tile, t);
            if (NEEDS) ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
            if (!ok) return;
            if (!SPLIT && NEEDS && lane == 0 && wanted) {
                fetch(0, mine, ready);
                if (wanted > 1) fetch(1, other, ready + 8);
            }
            for (uint32_t b = 0; b < max(wanted, 1u) && ok; ++b) {
                const uint32_t cb = cb0 + b, j0 = cb * 64, which = SPLIT ? 0 : b;
                unsigned char* const here = which ? other : mine;
                if (SPLIT && wanted && lane == 0) {              // what the last block left in here has gone
                    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    if (MODE == kPoly) fetch(b, mine, ready);
                }
                ok = (b || bar_wait(sum_full + 8 * (n & 1), (n / 2) & 1)) && (!wanted || !NEEDS || bar_wait(ready + 8 * which, done[which] & 1));
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok || !wanted) break;
                if (NEEDS) ++done[which];
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                F2 v[32];
                read_64(v, tmem + (n & 1) * 256 + (quarter * 32 << 16) + team * 128 + b * 64);
                // the row's own place on the diagonal, in the block of columns that holds it
                const bool diagonal = MODE <= kPoly && i / 64 == cb;
                const uint32_t own = i % 64;
                float mine_own = 0.f;
                if (MODE <= kPoly && cb / 2 == bi) {
#pragma unroll
                    for (uint32_t q = 0; q < 32; ++q) {
                        if (own == 2 * q) mine_own = lo(v[q]);
                        if (own == 2 * q + 1) mine_own = hi(v[q]);
                    }
                    mine_own *= kDown2;
                }
                if (MODE == kGram && diagonal) a.diag_a[t.diagonal + i] = mine_own;
                if (!NEEDS) {
#pragma unroll
                    for (int q = 0; q < 32; ++q) v[q] = mul(v[q], twice(kDown));
                } else if (MODE == kApply) {
                    const F2 keep = twice(kQ1 + __ldcg(a.diag_b + t.diagonal + i));
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) {
                        const uint4 h = *reinterpret_cast<const uint4*>(here + piece(lane, c));
                        const F2 e[4] = {pair_of(h.x), pair_of(h.y), pair_of(h.z), pair_of(h.w)};
#pragma unroll
                        for (uint32_t q = 0; q < 4; ++q) v[4 * c + q] = fma(v[4 * c + q], twice(kDown), mul(e[q], keep));
                    }
                } else {
                    const float* d = a.diag_a + t.diagonal;
                    const float di = __ldcg(d + i);
                    const F2 keep = twice(fmaf(kQ5, di, kQ3));
                    const float e_own = fmaf(kQ5, fmaf(di, di, mine_own), kQ3 * di);
                    if (!SPLIT && diagonal) a.diag_b[t.diagonal + i] = e_own;
                    mine_own = SPLIT ? (kQ1 + e_own) * kUp : 0.f;
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) {
                        const uint4 h = *reinterpret_cast<const uint4*>(here + piece(lane, c));
                        F2 e[4] = {pair_of(h.x), pair_of(h.y), pair_of(h.z), pair_of(h.w)};
                        if (SPLIT) {
                            const uint4 l = *reinterpret_cast<const uint4*>(other + piece(lane, c));
                            e[0] = add(e[0], pair_of(l.x)); e[1] = add(e[1], pair_of(l.y)); e[2] = add(e[2], pair_of(l.z)); e[3] = add(e[3], pair_of(l.w));
                        }
                        const float4 d0 = __ldcg(reinterpret_cast<const float4*>(d + j0 + 8 * c)), d1 = __ldcg(reinterpret_cast<const float4*>(d + j0 + 8 * c + 4));
                        const F2 dj[4] = {pair(d0.x, d0.y), pair(d0.z, d0.w), pair(d1.x, d1.y), pair(d1.z, d1.w)};
#pragma unroll
                        for (uint32_t q = 0; q < 4; ++q) v[4 * c + q] = fma(v[4 * c + q], twice(kQ5 * kDown), mul(e[q], fma(dj[q], twice(kQ5), keep)));
                    }
                }
                uint32_t h[32], low_h[SPLIT ? 32 : 1];
#pragma unroll
                for (int q = 0; q < 32; ++q) h[q] = half2_of(v[q]);
                if (SPLIT) {
#pragma unroll
                    for (int q = 0; q < 32; ++q) {               // what float16 leaves over
                        const F2 x = pair_of(h[q]);
                        low_h[q] = half2_of(pair(lo(v[q]) - lo(x), hi(v[q]) - hi(x)));
                    }
                }
#pragma unroll
                for (uint32_t c = 0; c < 8; ++c) {
                    *reinterpret_cast<uint4*>(here + piece(lane, c)) = make_uint4(h[4 * c], h[4 * c + 1], h[4 * c + 2], h[4 * c + 3]);
                    if (SPLIT) *reinterpret_cast<uint4*>(other + piece(lane, c)) = make_uint4(low_h[4 * c], low_h[4 * c + 1], low_h[4 * c + 2], low_h[4 * c + 3]);
                }
                if (diagonal) {                                  // none in A; in B with `split` alone, with the 3.4445 of X
                    const __half d = __float2half_rn(MODE == kPoly ? mine_own : 0.f);
                    *reinterpret_cast<__half*>(here + piece(lane, own / 8) + own % 8 * 2) = d;
                    if (SPLIT) *reinterpret_cast<__half*>(other + piece(lane, own / 8) + own % 8 * 2) = __float2half_rn(MODE == kPoly ? mine_own - __half2float(d) : 0.f);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    copy_out(out + (uint64_t)cb * kBlockBytes, smem_of(here), kRows);
                    if (SPLIT) copy_out(out + (uint64_t)cb * kBlockBytes + low, smem_of(other), kRows);
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
                if (MODE <= kPoly && cb / 2 < bi) {              // below the diagonal: the transpose too; lanes have neighbours, 64 bytes a store
                    unsigned char* const there = (MODE == kGram ? a.a : a.b) + (t.a_block + (uint64_t)(cb / 2) * 2 * t.mb + i / 64) * kBlockBytes + cb % 2 * (kBlockBytes / 2) + i % 8 * 2;
#pragma unroll
                    for (uint32_t q = 0; q < 64; ++q) {
                        *reinterpret_cast<uint16_t*>(there + piece(q, i % 64 / 8)) = (uint16_t)(q & 1 ? h[q / 2] >> 16 : h[q / 2]);
                        if (SPLIT) *reinterpret_cast<uint16_t*>(there + low + piece(q, i % 64 / 8)) = (uint16_t)(q & 1 ? low_h[q / 2] >> 16 : low_h[q / 2]);
                    }
                }
            }
            if (!ok) return;
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            if (MODE <= kPoly) asm volatile("fence.proxy.async;" ::: "memory");          // the transpose is read by copies
            __syncwarp();
            if (lane == 0) {
                bar_arrive_at(sum_empty + 8 * (n & 1), 0);       // the first block multiplies for both
                // all that this warp wrote is in place: the stores of its lanes before the barrier above, the copies after this wait
                asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
                asm volatile("fence.acq_rel.gpu;" ::: "memory");
                asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(a.written + MODE * a.n + tile.which) : "memory");
            }
            __syncwarp();
        };
        for (uint32_t u = our_pair; u < tiles && ok; u += pairs, ++n) {
            const Tile tile = tile_at(a, u);
            const PlanEntry t = entries[tile.which];
            if (tile.mode == kGram) finish(Mode<kGram>(), tile, t);
            else if (tile.mode == kPoly) finish(Mode<kPoly>(), tile, t);
            else finish(Mode<kApply>(), tile, t);
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        if (!ok && lane == 0) {
            words[1] = 1;
            for (uint32_t w = 0; w < 2; ++w) bar_wait(ready + 8 * w, done[w] & 1);       // copies that may be in flight
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cg::this_cluster().sync();                                   // neither block's memory goes before the other is done with it
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(words + 1)) *a.word = 1;
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ---- small matrices ----
//
// A matrix of at most 128 x 512 (128 x 256 with `split`; either way) goes through all its steps in one block's shared memory: X (up to 128 KB) and A,
// which B replaces, each product's sum in tensor memory, read out by eight warps. A chain of launches costs 10 us a product at any size (12 matrices
// of 64 x 64 and 64 x 256 in 32-bit products: 164 us a call in all, so 63: five steps of three dependent products, 46 us, which latency bounds).

constexpr uint32_t kSmallThreads = 256, kSmallBlocks = 8;                        // X's
constexpr uint32_t kSmallSmem = (kSmallBlocks + 4) * kBlockBytes + 1024 + 1536;

__device__ __forceinline__ void multiply_alone(uint32_t d, uint64_t a, uint64_t b, uint32_t how, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}

template <bool SPLIT> __global__ void __launch_bounds__(kSmallThreads, 1) muon_small_kernel(MuonArgs a) {
    extern __shared__ unsigned char raw[];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, quarter = warp & 3, half = warp >> 2, r = quarter * 32 + lane;
    unsigned char* const x = raw + (1024 - (smem_of(raw) & 1023)) % 1024;        // X's blocks, its low numbers', A's, its low numbers'
    constexpr uint32_t kLowX = kSmallBlocks / 2 * kBlockBytes, kLowA = 2 * kBlockBytes;
    unsigned char* const m = x + kSmallBlocks * kBlockBytes;
    float* const diag = reinterpret_cast<float*>(m + 2 * kLowA);                 // A's 128, B's 128 (with `split` in B)
    const uint32_t bar = smem_of(diag + 256);                                    // copies; products
    uint32_t* const words = reinterpret_cast<uint32_t*>(diag + 260);
    if (threadIdx.x == 0) {
        bar_init(bar, 1); bar_init(bar + 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
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
    bool ok = true;
    uint32_t copied = 0, multiplied = 0;
    const uint32_t count = isfinite(scale) ? a.items[kSmall] : 0;                // not by the word: another block may be setting it, and threads would part at a barrier
    // The block's products of `steps` blocks of 64 of the inner dimension; everybody waits for them.
    auto product = [&](const unsigned char* left, uint32_t left_low, const unsigned char* right, uint32_t right_low, uint32_t steps, uint32_t columns, bool along) {
        if (threadIdx.x == 0) {
            for (uint32_t c = 0; c < columns; c += 256) {        // right operands of at most 256 columns
                const uint32_t how = 1u << 4 | (along ? 1u << 16 : 0u) | min(256u, columns - c) / 8 << 17 | 128u / 16 << 24;
                for (uint32_t g = 0; g < (SPLIT ? 3 : 1); ++g)
                    for (uint32_t s = 0; s < steps; ++s)
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) {
                            const uint32_t l = smem_of(left) + (SPLIT && g == 1 ? left_low : 0) + s * kBlockBytes + k * 32, q = smem_of(right) + (SPLIT && g == 0 ? right_low : 0) + c / 64 * kBlockBytes;
                            multiply_alone(tmem + c, operand(l, 16, 1024), along ? operand(q + s * (kBlockBytes / 2) + k * 2048, kBlockBytes, 1024) : operand(q + s * kBlockBytes + k * 32, 16, 1024),
                                           how, g || s || k);
                        }
            }
            asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar + 8) : "memory");
        }
        __syncwarp();
        ok = !__syncthreads_or(!bar_wait(bar + 8, multiplied++ & 1));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    // 64 columns of the sum as 16-bit numbers into a block.
    auto put = [&](unsigned char* block, uint32_t low, const F2* v, float own_value, bool own) {
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c) {
            uint32_t h[4], l[4];
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                const F2 e = v[4 * c + q];
                h[q] = half2_of(e);
                if (SPLIT) { const F2 y = pair_of(h[q]); l[q] = half2_of(pair(lo(e) - lo(y), hi(e) - hi(y))); }
            }
            *reinterpret_cast<uint4*>(block + piece(r, c)) = make_uint4(h[0], h[1], h[2], h[3]);
            if (SPLIT) *reinterpret_cast<uint4*>(block + low + piece(r, c)) = make_uint4(l[0], l[1], l[2], l[3]);
        }
        if (own) {                                               // the row's place on the diagonal
            const uint32_t at = piece(r, r % 64 / 8) + r % 8 * 2;
            const __half h = __float2half_rn(own_value);
            *reinterpret_cast<__half*>(block + at) = h;
            if (SPLIT) *reinterpret_cast<__half*>(block + low + at) = __float2half_rn(own_value - __half2float(h));
        }
    };
    auto own_of = [&](const F2* v) {
        float y = 0.f;
#pragma unroll
        for (uint32_t q = 0; q < 32; ++q) {
            if (r % 64 == 2 * q) y = lo(v[q]);
            if (r % 64 == 2 * q + 1) y = hi(v[q]);
        }
        return y * kDown2;
    };
    auto written = [] {                                          // by threads, read by products and copies next
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    for (uint32_t u = blockIdx.x; u < count && ok; u += gridDim.x) {
        const PlanEntry t = plan_entries(a.plan)[a.maps[kSmall][u]];
        const uint32_t bytes = t.nb * kBlockBytes;
        if (threadIdx.x == 0) {
            const unsigned char* from = a.x[0] + t.x_block * kBlockBytes;
            bar_expect(bar, (SPLIT ? 2 : 1) * bytes);
            copy_in(smem_of(x), from, bytes, bar);
            if (SPLIT) copy_in(smem_of(x) + kLowX, from + a.x_bytes, bytes, bar);
        }
        ok = !__syncthreads_or(!bar_wait(bar, copied++ & 1));
        const bool own = r / 64 == half;
        for (uint32_t s = 0; s < a.steps && ok; ++s) {
            F2 v[32];
            product(x, kLowX, x, kLowX, t.nb, 128, false);
            if (!ok) break;
            read_64(v, tmem + (quarter * 32 << 16) + half * 64);
            if (own) diag[r] = own_of(v);
#pragma unroll
            for (int q = 0; q < 32; ++q) v[q] = mul(v[q], twice(kDown));
            put(m + half * kBlockBytes, kLowA, v, 0.f, own);
            written();
            product(m, kLowA, m, kLowA, t.kb, 128, false);
            if (!ok) break;
            read_64(v, tmem + (quarter * 32 << 16) + half * 64);
            const float di = diag[r], more = own ? own_of(v) : 0.f;
            const F2 keep = twice(fmaf(kQ5, di, kQ3));
            unsigned char* const block = m + half * kBlockBytes;
#pragma unroll
            for (uint32_t c = 0; c < 8; ++c) {
                const uint4 h = *reinterpret_cast<const uint4*>(block + piece(r, c));
                F2 e[4] = {pair_of(h.x), pair_of(h.y), pair_of(h.z), pair_of(h.w)};
                if (SPLIT) {
                    const uint4 l = *reinterpret_cast<const uint4*>(block + kLowA + piece(r, c));
                    e[0] = add(e[0], pair_of(l.x)); e[1] = add(e[1], pair_of(l.y)); e[2] = add(e[2], pair_of(l.z)); e[3] = add(e[3], pair_of(l.w));
                }
                const float4 d0 = *reinterpret_cast<const float4*>(diag + half * 64 + 8 * c), d1 = *reinterpret_cast<const float4*>(diag + half * 64 + 8 * c + 4);
                const F2 dj[4] = {pair(d0.x, d0.y), pair(d0.z, d0.w), pair(d1.x, d1.y), pair(d1.z, d1.w)};
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) v[4 * c + q] = fma(v[4 * c + q], twice(kQ5 * kDown), mul(e[q], fma(dj[q], twice(kQ5), keep)));
            }
            const float e_own = fmaf(kQ5, fmaf(di, di, more), kQ3 * di);
            if (!SPLIT && own) diag[128 + r] = e_own;
            put(block, kLowA, v, SPLIT ? (kQ1 + e_own) * kUp : 0.f, own);
            written();
            product(m, kLowA, x, kLowX, t.kb, t.nb * 64, true);
            if (!ok) break;
            for (uint32_t q = half; q < t.nb; q += 2) {
                read_64(v, tmem + (quarter * 32 << 16) + q * 64);
                if (SPLIT) {
#pragma unroll
                    for (int p = 0; p < 32; ++p) v[p] = mul(v[p], twice(kDown));
                } else {
                    const F2 keep_x = twice(kQ1 + diag[128 + r]);
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) {
                        const uint4 h = *reinterpret_cast<const uint4*>(x + q * kBlockBytes + piece(r, c));
                        const F2 e[4] = {pair_of(h.x), pair_of(h.y), pair_of(h.z), pair_of(h.w)};
#pragma unroll
                        for (uint32_t p = 0; p < 4; ++p) v[4 * c + p] = fma(v[4 * c + p], twice(kDown), mul(e[p], keep_x));
                    }
                }
                put(x + q * kBlockBytes, kLowX, v, 0.f, false);
            }
            written();
        }
        if (threadIdx.x == 0 && ok) {
            unsigned char* to = a.x[a.steps & 1] + t.x_block * kBlockBytes;
            copy_out(to, smem_of(x), bytes);
            if (SPLIT) copy_out(to + a.x_bytes, smem_of(x) + kLowX, bytes);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        }
    }
    if (threadIdx.x == 0 && !ok) {                               // a wait has given up: once more, for what may still be on its way
        *a.word = 1;
        bar_wait(bar, (copied - 1) & 1);
        if (multiplied) bar_wait(bar + 8, (multiplied - 1) & 1);
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <bool SPLIT> static cudaError_t small(const MuonArgs& a, int sms, cudaStream_t st) {
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3(a.items[kSmall] < (uint32_t)sms ? a.items[kSmall] : (uint32_t)sms); how.blockDim = dim3(kSmallThreads); how.dynamicSmemBytes = kSmallSmem;
    how.stream = st; how.attrs = &early; how.numAttrs = 1;
    return cudaLaunchKernelEx(&how, muon_small_kernel<SPLIT>, a);
}

// All steps' products in one cooperative launch: as many pairs as the GPU holds at once, since tiles wait for those of other pairs.
template <bool SPLIT> static cudaError_t products(const MuonArgs& a, int most, cudaStream_t st) {
    const uint32_t busiest = a.items[kGramTiles] > a.items[kApplyTiles] ? a.items[kGramTiles] : a.items[kApplyTiles];      // no more pairs than a product has tiles
    cudaLaunchAttribute at_once{};
    at_once.id = cudaLaunchAttributeCooperative;
    at_once.val.cooperative = 1;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3(2 * (busiest < (uint32_t)most ? busiest : (uint32_t)most)); how.blockDim = dim3(kProductThreads); how.dynamicSmemBytes = kProductSmem;
    how.stream = st; how.attrs = &at_once; how.numAttrs = 1;
    return cudaLaunchKernelEx(&how, muon_products_kernel<SPLIT>, a);
}

// Whether the GPU can run the kernels that take most of its shared memory; `most`: how many pairs of blocks it holds at once.
template <bool SPLIT> static cudaError_t ready(const MuonArgs& a, int& most) {
    cudaError_t e = cudaSuccess;
    if (a.items[kSmall]) e = cudaFuncSetAttribute(muon_small_kernel<SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmem);
    if (e != cudaSuccess || !a.items[kGramTiles]) return e;
    if ((e = cudaFuncSetAttribute(muon_products_kernel<SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem)) != cudaSuccess) return e;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3(2); how.blockDim = dim3(kProductThreads); how.dynamicSmemBytes = kProductSmem;
    if ((e = cudaOccupancyMaxActiveClusters(&most, muon_products_kernel<SPLIT>, &how)) != cudaSuccess) return e;
    return most < 1 ? cudaErrorInvalidConfiguration : cudaSuccess;
}

template <bool SPLIT> static cudaError_t step(const MuonArgs& a, int sms, cudaStream_t st) {
    int most = 0;
    cudaError_t e = ready<SPLIT>(a, most);                       // before the momentum moves: it moves in place, and once
    if (e != cudaSuccess) return e;
    muon_momentum_kernel<<<a.items[kChunks], 256, 0, st>>>(a);
    e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_second(muon_norm_kernel, a.n, 256, st, a);
    if (e == cudaSuccess) e = launch_second(muon_layout_kernel, a.items[kBlocks], 256, st, a);
    if (e == cudaSuccess && a.items[kSmall]) e = small<SPLIT>(a, sms, st);
    if (e == cudaSuccess && a.items[kGramTiles]) e = products<SPLIT>(a, most, st);
    if (e == cudaSuccess) e = launch_second(muon_update_kernel, a.items[kBlocks], 256, st, a);
    return e;
}

cudaError_t launch_muon(const MuonArgs& a, int sms, cudaStream_t st) { return a.split ? step<true>(a, sms, st) : step<false>(a, sms, st); }

}  // namespace ftc
