// The norm of all gradients and the AdamW step, over a table of tensors. A warp takes one block of FTC_STATE_BLOCK elements of one
// tensor at a time, 8 elements a lane; the table gives it the block's tensor.
//
// A block is read in one of two layouts. Wide: lane l holds the elements 8 l .. 8 l + 7, one load of 32 (or 16) bytes for each array;
// it takes a full block of a tensor whose arrays all begin on such boundaries. Narrow: lane l holds the elements l, l + 32, ..., one
// element a load, each load of the warp one contiguous run: for any alignment and for a tensor's last block.
#include "ftc_train.cuh"

namespace ftc {

constexpr uint32_t kWarps = 8;
constexpr float kTiny = 1.1754943508222875e-38f;                 // 2^-126, the smallest scale
constexpr float kInv127 = 1.0f / 16129.0f, kInv255 = 1.0f / 65025.0f;

struct Raw { uint32_t r[8]; };                                   // 8 elements as loaded: numbers are made of them once all loads are out

__device__ __forceinline__ void load_32(const void* p, uint32_t* r) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store_32(void* p, const uint32_t* r) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void load_16(const void* p, uint32_t* r) {
    const uint4 v = *static_cast<const uint4*>(p);
    r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
}

// Which elements a lane holds of the block that begins at element e0 of a tensor of n.
template <bool WIDE> __device__ __forceinline__ uint32_t at(uint32_t lane, int j) { return WIDE ? lane * 8 + j : j * 32 + lane; }

template <bool WIDE> __device__ __forceinline__ void load_raw(Raw& x, const void* base, uint32_t dtype, uint64_t e0, uint32_t lane, uint32_t left) {
    if (WIDE) {
        if (dtype == FTC_F32) load_32(static_cast<const float*>(base) + e0 + lane * 8, x.r);
        else load_16(static_cast<const uint16_t*>(base) + e0 + lane * 8, x.r);
        return;
    }
    if (dtype == FTC_F32) {
        const uint32_t* p = static_cast<const uint32_t*>(base) + e0;
#pragma unroll
        for (int j = 0; j < 8; ++j) x.r[j] = at<WIDE>(lane, j) < left ? p[at<WIDE>(lane, j)] : 0u;
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(base) + e0;
#pragma unroll
        for (int j = 0; j < 8; ++j) x.r[j] = at<WIDE>(lane, j) < left ? p[at<WIDE>(lane, j)] : 0u;
    }
}

__device__ __forceinline__ float half_f32(uint32_t bits) { return __half2float(__ushort_as_half((unsigned short)bits)); }

template <bool WIDE> __device__ __forceinline__ void numbers(float* v, const Raw& x, uint32_t dtype) {
    if (dtype == FTC_F32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(x.r[j]);
    } else if (dtype == FTC_BF16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(WIDE ? (j & 1 ? x.r[j / 2] & 0xFFFF0000u : x.r[j / 2] << 16) : x.r[j] << 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = half_f32(WIDE ? (j & 1 ? x.r[j / 2] >> 16 : x.r[j / 2] & 0xFFFFu) : x.r[j]);
    }
}

// Elements whose bit in `live` is set; all of them in the wide layout if all bits are.
template <bool WIDE> __device__ __forceinline__ void store_numbers(void* base, uint32_t dtype, uint64_t e0, uint32_t lane, const float* v, uint32_t live) {
    uint32_t r[8];
    if (WIDE && live == 0xFFu) {
        if (dtype == FTC_F32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(v[j]);
            store_32(static_cast<float*>(base) + e0 + lane * 8, r);
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (dtype == FTC_BF16) { const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]); r[j] = *reinterpret_cast<const uint32_t*>(&p); }
            else { const __half2 p = __floats2half2_rn(v[2 * j], v[2 * j + 1]); r[j] = *reinterpret_cast<const uint32_t*>(&p); }
        }
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + e0 + lane * 8) = make_uint4(r[0], r[1], r[2], r[3]);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (live >> j & 1u) {
            const uint64_t i = e0 + at<WIDE>(lane, j);
            if (dtype == FTC_F32) static_cast<float*>(base)[i] = v[j];
            else if (dtype == FTC_BF16) static_cast<__nv_bfloat16*>(base)[i] = from_f32<__nv_bfloat16>(v[j]);
            else static_cast<__half*>(base)[i] = from_f32<__half>(v[j]);
        }
}

__device__ __forceinline__ uint2 record(const TableEntry& t, uint64_t message) {
    return *reinterpret_cast<const uint2*>(t.status + message * FTC_STATUS_WORDS);
}
// 1 / processes included, 0 where the message was not delivered.
__device__ __forceinline__ float share_of(uint2 s) { return (s.x & 0xFFu) == FTC_ST_OK && s.y ? 1.f / (float)s.y : 0.f; }

// What each of the lane's elements is multiplied with, and which were delivered (bits). One division where the lane's elements are
// neighbours; elements and messages of more than 32 bits take the long one.
template <bool WIDE> __device__ __forceinline__ uint32_t shares(float* w, const TableEntry& t, uint64_t e0, uint32_t lane, uint32_t left) {
    uint32_t live = 0;
    if (!t.status) {
#pragma unroll
        for (int j = 0; j < 8; ++j) { w[j] = 1.f; live |= (WIDE || at<WIDE>(lane, j) < left ? 1u : 0u) << j; }
        return live;
    }
    const bool small = e0 + FTC_STATE_BLOCK <= 0xFFFFFFFFull;
    if (WIDE) {
        const uint64_t e = e0 + lane * 8;
        uint64_t q = small ? (uint32_t)e / t.k : e / t.k;
        uint32_t r = (uint32_t)(e - q * t.k);
        float s = share_of(record(t, q));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = s;
            live |= (s > 0.f ? 1u : 0u) << j;
            if (j < 7 && ++r == t.k) { r = 0; s = share_of(record(t, ++q)); }
        }
        return live;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        w[j] = 0.f;
        if (at<WIDE>(lane, j) < left) {
            const uint64_t e = e0 + at<WIDE>(lane, j);
            w[j] = share_of(record(t, small ? (uint32_t)e / t.k : e / t.k));
            live |= (w[j] > 0.f ? 1u : 0u) << j;
        }
    }
    return live;
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
__device__ __forceinline__ float warp_max_bits(uint32_t v) { return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, v)); }

template <int BITS, bool WIDE>
__device__ __forceinline__ void adamw_block(const AdamArgs& a, const TableEntry& t, uint64_t b, uint32_t lane, uint64_t e0, uint32_t left, float scale) {
    Raw gr, pr, mr, vr;
    const uint32_t pd = t.master ? (uint32_t)FTC_F32 : t.param_dtype;
    void* weights = t.master ? t.master : t.param;
    load_raw<WIDE>(gr, t.grad, t.grad_dtype, e0, lane, left);
    load_raw<WIDE>(pr, weights, pd, e0, lane, left);
    const uint64_t q = b * FTC_STATE_BLOCK;
    float ms = 0.f, vs = 0.f;
    if (BITS == 32) {
        load_raw<WIDE>(mr, a.m, FTC_F32, q, lane, FTC_STATE_BLOCK);
        load_raw<WIDE>(vr, a.v, FTC_F32, q, lane, FTC_STATE_BLOCK);
    } else {
        const uint8_t *mp = static_cast<const uint8_t*>(a.m) + q, *vp = static_cast<const uint8_t*>(a.v) + q;
        if (WIDE) {
            const uint2 x = reinterpret_cast<const uint2*>(mp)[lane], y = reinterpret_cast<const uint2*>(vp)[lane];
            mr.r[0] = x.x; mr.r[1] = x.y; vr.r[0] = y.x; vr.r[1] = y.y;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) { mr.r[j] = mp[j * 32 + lane]; vr.r[j] = vp[j * 32 + lane]; }
        }
        ms = a.m_scale[b]; vs = a.v_scale[b];
    }
    float w[8], g[8], p[8], m[8], v[8];
    const uint32_t live = shares<WIDE>(w, t, e0, lane, left);
    numbers<WIDE>(g, gr, t.grad_dtype);
    numbers<WIDE>(p, pr, pd);
    if (BITS == 32) { numbers<true>(m, mr, FTC_F32); numbers<true>(v, vr, FTC_F32); }
    else {
        ms *= kInv127; vs *= kInv255;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t cm = WIDE ? mr.r[j / 4] >> (j % 4 * 8) & 0xFFu : mr.r[j], cv = WIDE ? vr.r[j / 4] >> (j % 4 * 8) & 0xFFu : vr.r[j];
            const float c = (float)(int8_t)cm, d = (float)cv, r = d * d * vs;
            m[j] = c * fabsf(c) * ms;
            v[j] = r * r;
        }
    }
    const float lr = a.lr * t.lr_scale, keep = 1.f - lr * t.weight_decay, rate = lr * a.fix1;
    float root[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float gj = g[j] * w[j] * scale, mj = m[j] * a.beta1 + gj * a.rest1, vj = v[j] * a.beta2 + gj * gj * a.rest2;
        root[j] = sqrtf(vj);
        const float pj = p[j] * keep - mj / (root[j] * a.fix2 + a.eps) * rate;
        if (live >> j & 1u) { m[j] = mj; v[j] = vj; p[j] = pj; }
        else if (BITS == 8) root[j] = sqrtf(v[j]);
    }
    store_numbers<WIDE>(weights, pd, e0, lane, p, live);
    if (t.master) store_numbers<WIDE>(t.param, t.param_dtype, e0, lane, p, live);
    if (BITS == 32) {
        store_numbers<WIDE>(a.m, FTC_F32, q, lane, m, live);
        store_numbers<WIDE>(a.v, FTC_F32, q, lane, v, live);
        return;
    }
    if (!__any_sync(0xFFFFFFFFu, live)) return;
    uint32_t mm = 0, rm = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        mm = max(mm, __float_as_uint(m[j]) & 0x7FFFFFFFu);
        rm = max(rm, __float_as_uint(root[j]) & 0x7FFFFFFFu);
    }
    ms = warp_max_bits(mm); vs = warp_max_bits(rm);
    ms = ms < kTiny ? kTiny : ms; vs = vs < kTiny ? kTiny : vs;             // NaN stays
    const float mi = 1.f / ms, vi = 1.f / vs;
    uint32_t cm[8], cv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float c = nearest_root(fabsf(m[j]) * mi * 16129.f, 127.f);
        float d = nearest_root(root[j] * vi * 65025.f, 255.f);
        if (root[j] > 0.f) d = fmaxf(d, 1.f);
        cm[j] = (uint32_t)(int)(m[j] < 0.f ? -c : c) & 0xFFu;
        cv[j] = (uint32_t)d;
    }
    uint8_t *mp = static_cast<uint8_t*>(a.m) + q, *vp = static_cast<uint8_t*>(a.v) + q;
    if (WIDE) {
        reinterpret_cast<uint2*>(mp)[lane] = make_uint2(cm[0] | cm[1] << 8 | cm[2] << 16 | cm[3] << 24, cm[4] | cm[5] << 8 | cm[6] << 16 | cm[7] << 24);
        reinterpret_cast<uint2*>(vp)[lane] = make_uint2(cv[0] | cv[1] << 8 | cv[2] << 16 | cv[3] << 24, cv[4] | cv[5] << 8 | cv[6] << 16 | cv[7] << 24);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) { mp[j * 32 + lane] = (uint8_t)cm[j]; vp[j * 32 + lane] = (uint8_t)cv[j]; }
    }
    if (lane == 0) { a.m_scale[b] = ms; a.v_scale[b] = vs; }
}

template <int BITS>
__global__ void __launch_bounds__(kWarps * 32) adamw_kernel(AdamArgs a) {
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t b = blockIdx.x * (uint64_t)kWarps + (threadIdx.x >> 5);
    if (b >= a.n_blocks) return;
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    const TableEntry t = table_entries(a.table)[table_map(a.table, a.n_params)[b]];
    if (!isfinite(scale)) return;
    const uint64_t e0 = (b - t.first_block) * FTC_STATE_BLOCK, left = t.n - e0;
    if (t.wide && left >= FTC_STATE_BLOCK) adamw_block<BITS, true>(a, t, b, lane, e0, FTC_STATE_BLOCK, scale);
    else adamw_block<BITS, false>(a, t, b, lane, e0, left < FTC_STATE_BLOCK ? (uint32_t)left : FTC_STATE_BLOCK, scale);
}

cudaError_t launch_adamw(const AdamArgs& a, int, cudaStream_t st) {
    const uint32_t grid = (uint32_t)((a.n_blocks + kWarps - 1) / kWarps);
    if (a.bits == 32) adamw_kernel<32><<<grid, kWarps * 32, 0, st>>>(a);
    else adamw_kernel<8><<<grid, kWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}

// A lane reads 8 codes of each state (8 bytes) and writes 32 bytes of each output.
__global__ void __launch_bounds__(256) adamw_states_kernel(uint64_t blocks, const uint8_t* m, const uint8_t* v, const float* ms, const float* vs, float* mo, float* vo) {
    const uint64_t i = blockIdx.x * 256ull + threadIdx.x, b = i / 32;
    if (b >= blocks) return;
    const uint2 x = reinterpret_cast<const uint2*>(m)[i], y = reinterpret_cast<const uint2*>(v)[i];
    const float sm = ms[b] * kInv127, sv = vs[b] * kInv255;
    uint32_t rm[8], rv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t cm = (j < 4 ? x.x : x.y) >> (j % 4 * 8) & 0xFFu, cv = (j < 4 ? y.x : y.y) >> (j % 4 * 8) & 0xFFu;
        const float c = (float)(int8_t)cm, d = (float)cv, r = d * d * sv;
        rm[j] = __float_as_uint(c * fabsf(c) * sm);
        rv[j] = __float_as_uint(r * r);
    }
    store_32(mo + i * 8, rm);
    store_32(vo + i * 8, rv);
}

cudaError_t launch_adamw_states(uint64_t blocks, const void* m, const void* v, const float* ms, const float* vs, float* mo, float* vo, int, cudaStream_t st) {
    adamw_states_kernel<<<(uint32_t)((blocks + 7) / 8), 256, 0, st>>>(blocks, static_cast<const uint8_t*>(m), static_cast<const uint8_t*>(v), ms, vs, mo, vo);
    return cudaGetLastError();
}

// ---- the norm: warp w adds up the squares of the blocks [w*span, (w+1)*span) and leaves one sum for each tensor it meets; warp w and
// tensor t share slot w + t (going on by one block either grows, so no two pairs with blocks in common share a slot)

constexpr int kAhead = 4;                                        // blocks whose loads a warp has out at once

template <bool WIDE> __device__ __forceinline__ double block_squares(const Raw& x, const TableEntry& t, uint64_t e0, uint32_t lane, uint32_t left) {
    float w[8], g[8];
    numbers<WIDE>(g, x, t.grad_dtype);
    double s = 0;
    if (t.status) {
        const uint32_t live = shares<WIDE>(w, t, e0, lane, left);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = live >> j & 1u ? g[j] * w[j] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fma((double)g[j], (double)g[j], s);       // elements behind the end were loaded as zeros
    return s;
}

__global__ void __launch_bounds__(kWarps * 32) grad_squares_kernel(const void* table, uint32_t n_params, uint64_t n_blocks, uint64_t span, double* slots) {
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t w = blockIdx.x * (uint64_t)kWarps + (threadIdx.x >> 5);
    uint64_t b = w * span;
    const uint64_t b1 = b + span < n_blocks ? b + span : n_blocks;
    while (b < b1) {
        const uint32_t ti = table_map(table, n_params)[b];
        const TableEntry t = table_entries(table)[ti];
        const uint64_t last = t.first_block + (t.n + FTC_STATE_BLOCK - 1) / FTC_STATE_BLOCK, end = last < b1 ? last : b1;
        const uint64_t whole = t.wide ? t.first_block + t.n / FTC_STATE_BLOCK : 0, end_wide = whole < end ? whole : end;
        double s = 0;
        for (; b + kAhead <= end_wide; b += kAhead) {
            Raw x[kAhead];
            const uint64_t e0 = (b - t.first_block) * FTC_STATE_BLOCK;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load_raw<true>(x[i], t.grad, t.grad_dtype, e0 + i * FTC_STATE_BLOCK, lane, FTC_STATE_BLOCK);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) s += block_squares<true>(x[i], t, e0 + i * FTC_STATE_BLOCK, lane, FTC_STATE_BLOCK);
        }
        for (; b < end; ++b) {
            Raw x;
            const uint64_t e0 = (b - t.first_block) * FTC_STATE_BLOCK, rest = t.n - e0;
            const uint32_t left = rest < FTC_STATE_BLOCK ? (uint32_t)rest : FTC_STATE_BLOCK;
            load_raw<false>(x, t.grad, t.grad_dtype, e0, lane, left);
            s += block_squares<false>(x, t, e0, lane, left);
        }
        s = warp_sum(s);
        if (lane == 0) slots[w + ti] = s;
    }
}

// One block: a warp for each tensor's sum, then the sum over tensors.
__global__ void __launch_bounds__(1024) grad_norm_kernel(const void* table, uint32_t n_params, uint64_t span, float max_norm, const double* slots, double* sums,
                                                         float* norm, float* norms) {
    __shared__ double part[32];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t ti = warp; ti < n_params; ti += 32) {
        const uint64_t n = table_entries(table)[ti].n, first = table_entries(table)[ti].first_block;
        double s = 0;
        if (n) {
            const uint64_t last = first + (n - 1) / FTC_STATE_BLOCK;
#pragma unroll 8
            for (uint64_t w = first / span + lane; w <= last / span; w += 32) s += slots[w + ti];
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
    const uint64_t cap = (uint64_t)sm_count * 32;
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
