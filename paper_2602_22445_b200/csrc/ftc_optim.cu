// The norm of all gradients and the AdamW step, over a table of tensors. A warp takes one block of FTC_STATE_BLOCK elements of one
// tensor at a time, 8 elements a lane; the table gives it the block's tensor.
//
// A block is read in one of two layouts. Wide: lane l holds the elements 8 l .. 8 l + 7, one load of 32 (or 16) bytes for each array;
// it takes a full block of a tensor whose arrays all begin on such boundaries. Narrow: lane l holds the elements l, l + 32, ..., one
// element a load, each load of the warp one contiguous run: for any alignment and for a tensor's last block.
#include "ftc_f32x2.cuh"
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

template <typename U> __device__ __forceinline__ void load_narrow(Raw& x, const U* p, uint32_t lane, uint32_t left) {
    if (left >= FTC_STATE_BLOCK) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.r[j] = p[j * 32];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.r[j] = lane + j * 32 < left ? p[j * 32] : 0u;
    }
}
template <bool WIDE> __device__ __forceinline__ void load_raw(Raw& x, const void* base, uint32_t dtype, uint64_t e0, uint32_t lane, uint32_t left) {
    if (WIDE) {
        if (dtype == FTC_F32) load_32(static_cast<const float*>(base) + e0 + lane * 8, x.r);
        else load_16(static_cast<const uint16_t*>(base) + e0 + lane * 8, x.r);
        return;
    }
    if (dtype == FTC_F32) load_narrow(x, static_cast<const uint32_t*>(base) + e0 + lane, lane, left);
    else load_narrow(x, static_cast<const uint16_t*>(base) + e0 + lane, lane, left);
}

__device__ __forceinline__ float half_f32(uint32_t bits) { return __half2float(__ushort_as_half((unsigned short)bits)); }

template <bool WIDE> __device__ __forceinline__ void numbers(F2* v, const Raw& x, uint32_t dtype) {
    if (dtype == FTC_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair(__uint_as_float(x.r[2 * i]), __uint_as_float(x.r[2 * i + 1]));
    } else if (dtype == FTC_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = WIDE ? pair(__uint_as_float(x.r[i] << 16), __uint_as_float(x.r[i] & 0xFFFF0000u))
                        : pair(__uint_as_float(x.r[2 * i] << 16), __uint_as_float(x.r[2 * i + 1] << 16));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = WIDE ? pair(half_f32(x.r[i] & 0xFFFFu), half_f32(x.r[i] >> 16)) : pair(half_f32(x.r[2 * i]), half_f32(x.r[2 * i + 1]));
    }
}

// Elements whose bit in `live` is set; all of them in the wide layout if all bits are.
template <bool WIDE> __device__ __forceinline__ void store_numbers(void* base, uint32_t dtype, uint64_t e0, uint32_t lane, const F2* v, uint32_t live) {
    uint32_t r[8];
    if (WIDE && live == 0xFFu) {
        if (dtype == FTC_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { r[2 * i] = __float_as_uint(lo(v[i])); r[2 * i + 1] = __float_as_uint(hi(v[i])); }
            store_32(static_cast<float*>(base) + e0 + lane * 8, r);
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (dtype == FTC_BF16) { const __nv_bfloat162 p = __floats2bfloat162_rn(lo(v[i]), hi(v[i])); r[i] = *reinterpret_cast<const uint32_t*>(&p); }
            else { const __half2 p = __floats2half2_rn(lo(v[i]), hi(v[i])); r[i] = *reinterpret_cast<const uint32_t*>(&p); }
        }
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + e0 + lane * 8) = make_uint4(r[0], r[1], r[2], r[3]);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (live >> j & 1u) {
            const uint32_t i = at<WIDE>(lane, j);
            const float x = j & 1 ? hi(v[j / 2]) : lo(v[j / 2]);
            if (dtype == FTC_F32) (static_cast<float*>(base) + e0)[i] = x;
            else if (dtype == FTC_BF16) (static_cast<__nv_bfloat16*>(base) + e0)[i] = from_f32<__nv_bfloat16>(x);
            else (static_cast<__half*>(base) + e0)[i] = from_f32<__half>(x);
        }
}

__device__ __forceinline__ uint2 record(const TableEntry& t, uint64_t message) {
    return *reinterpret_cast<const uint2*>(t.status + message * FTC_STATUS_WORDS);
}
// 1 / processes included, 0 where the message was not delivered.
__device__ __forceinline__ float share_of(uint2 s) { return (s.x & 0xFFu) == FTC_ST_OK && s.y ? 1.f / (float)s.y : 0.f; }

// The message of element e, and its place in there. Messages of a power of two elements take a shift; elements of more than 32 bits the long
// division.
__device__ __forceinline__ uint64_t message_of(const TableEntry& t, uint64_t e, uint32_t& place) {
    if (t.k_shift != 255) { place = (uint32_t)e & (t.k - 1); return e >> t.k_shift; }
    const uint64_t q = e <= 0xFFFFFFFFull ? (uint32_t)e / t.k : e / t.k;
    place = (uint32_t)(e - q * t.k);
    return q;
}

// What each of the lane's elements is multiplied with, and which were delivered (bits).
template <bool WIDE> __device__ __forceinline__ uint32_t shares(F2* w, const TableEntry& t, uint64_t e0, uint32_t lane, uint32_t left) {
    uint32_t live = 0, r;
    float f[8];
    if (WIDE) {                                                      // neighbours: one division
        uint64_t q = message_of(t, e0 + lane * 8, r);
        float s = share_of(record(t, q));
        if (t.k - r >= 8) {                                          // one message has all eight
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = twice(s);
            return s > 0.f ? 0xFFu : 0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = s;
            live |= (s > 0.f ? 1u : 0u) << j;
            if (j < 7 && ++r == t.k) { r = 0; s = share_of(record(t, ++q)); }
        }
    } else if (t.k >= 3) {                                           // the block's messages, at most 87, over the lanes of the warp
        const uint64_t q = message_of(t, e0, r);
        const uint32_t last = (r + left - 1) / t.k, more = 32 / t.k, over = 32 - more * t.k;
        float s[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) s[i] = lane + i * 32 <= last ? share_of(record(t, q + lane + i * 32)) : 0.f;
        uint32_t m = (r + lane) / t.k, place = r + lane - m * t.k;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = __shfl_sync(0xFFFFFFFFu, s[0], m & 31), b = __shfl_sync(0xFFFFFFFFu, s[1], m & 31), c = __shfl_sync(0xFFFFFFFFu, s[2], m & 31);
            f[j] = m < 32 ? a : m < 64 ? b : c;
            if (at<WIDE>(lane, j) >= left) f[j] = 0.f;
            live |= (f[j] > 0.f ? 1u : 0u) << j;
            m += more; place += over;
            if (place >= t.k) { place -= t.k; ++m; }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = at<WIDE>(lane, j) < left ? share_of(record(t, message_of(t, e0 + at<WIDE>(lane, j), r))) : 0.f;
            live |= (f[j] > 0.f ? 1u : 0u) << j;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pair(f[2 * i], f[2 * i + 1]);
    return live;
}
template <bool WIDE> __device__ __forceinline__ uint32_t inside(uint32_t lane, uint32_t left) {
    if (WIDE) return 0xFFu;
    uint32_t live = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) live |= (at<WIDE>(lane, j) < left ? 1u : 0u) << j;
    return live;
}

// Byte j of the words x, and the numbers' low bytes back: a whole number c with |c| < 2^22 stands in the low bits of 3 * 2^22 + c
// (no conversion instructions, which run at a quarter of the rate).
constexpr float kWhole = 12582912.f;
__device__ __forceinline__ F2 bytes_numbers(uint32_t a, uint32_t b, F2 less) {                     // a, b: 2^23 + a byte, as bits
    return add(pair(__uint_as_float(a), __uint_as_float(b)), less);
}
__device__ __forceinline__ uint32_t byte_of(uint32_t w, int j) { return __byte_perm(w, 0x4B000000u, 0x7440 + j); }

__device__ __forceinline__ float one_above(float x) { float r; asm("set.gt.f32.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(x)); return r; }       // 1 where x > 0, else 0

// Largest size of three numbers; NaN where one of them is.
__device__ __forceinline__ float largest(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

__device__ __forceinline__ float smallest(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The whole numbers c nearest to sqrt(x), (c - 1/2)^2 <= x < (c + 1/2)^2, at most `most`, from an approximate root. The root and
// x may be off by some units in the last place: `far` collects how far the root lies from its whole number, and where that comes
// too near a half, c may be wrong. What counts is the distance from the exact root of the x that plain float32 gives. m has that x: the approximate
// root, good to 2^-23, is off by 127 * 2^-23 < 1.6e-5. v has it from an approximate root and two products, where plain float32 rounds its root
// and the same products: 2^-23 + 2^-24 and 4 * 2^-24 apart at most, half of which is left under the next root, which adds its own 2^-23:
// 255 * 2.75 * 2^-23 < 8.4e-5.
constexpr float kDoubtM = 2e-5f, kDoubtV = 9e-5f;
__device__ __forceinline__ float fast_root(float x) { float r; asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
// The same where x may be a subnormal number (second moments of gradients below 1e-18).
__device__ __forceinline__ float fast_root_of_any(float x) { float r; asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ F2 likely_roots(F2 x, float& far) {
    const F2 s = pair(fast_root(lo(x)), fast_root(hi(x))), c = add(add(s, twice(kWhole)), twice(-kWhole)), f = fma(c, twice(-1.f), s);
    far = largest(far, lo(f), hi(f));
    return c;
}
// The same without doubt: x - c^2 is exact in float32 (a multiple of x's last place, smaller than x), so two comparisons decide.
__device__ __noinline__ float nearest_root(float x, float most) {
    float c = floorf(__fsqrt_rn(x) + 0.5f);
    const float d = __fmaf_rn(-c, c, x);
    if (d >= c + 0.25f) c += 1.f;
    else if (d < 0.25f - c) c -= 1.f;
    return fminf(fmaxf(c, 0.f), most);                               // at c = 0 the lower comparison says nothing
}

// The whole number c below sqrt(x) or the one above, so that over many u from [0, 1) what they stand for is x on average (FOURTH: x^2, as
// v goes with the fourth power of its code): c + 1 where x lies more than u of the way. less_u: -u. A root beside a whole number may give the c
// below it, or the one above: the way is then a little over 1, or under 0, and the code that number all the same.
template <bool FOURTH> __device__ __forceinline__ F2 dithered_roots(F2 x, F2 less_u, float most) {
    const F2 r = pair(fast_root(lo(x)), fast_root(hi(x))), c = add(add(add(r, twice(-0.5f)), twice(kWhole)), twice(-kWhole));
    const F2 s = mul(c, c), d = fma(s, twice(-1.f), x), w = fma(c, twice(2.f), twice(1.f));             // s exact, w = (c+1)^2 - c^2
    const F2 more = FOURTH ? fma(less_u, mul(w, fma(s, twice(2.f), w)), mul(d, add(x, s))) : fma(less_u, w, d);   // (c+1)^4 - c^4 = w ((c+1)^2 + c^2)
    const F2 q = add(c, pair(one_above(lo(more)), one_above(hi(more))));
    return pair(fminf(lo(q), most), fminf(hi(q), most));
}
// -u of place e.
__device__ __forceinline__ float dither(uint32_t e, uint32_t phase) { return 1.f - __uint_as_float((e * kDitherPlace + phase) >> 9 | 0x3F800000u); }

// Largest of the warp's non-negative values, as bit patterns: infinities above all numbers, NaN above them.
__device__ __forceinline__ float warp_max_bits(uint32_t v) { return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, v)); }

// For divisors that eps keeps far above the smallest normal number.
__device__ __forceinline__ float fast_inverse(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }


// What a block needs, as loaded.
struct BlockIn { Raw gr, pr, mr, vr; float ms, vs; uint2 st; };
// Do a lane's eight neighbours have one record, found by a shift? It is loaded with the rest then.
__device__ __forceinline__ bool one_record(const TableEntry& t) { return t.k_shift >= 3 && t.k_shift != 255; }

template <int BITS, bool WIDE>
__device__ __forceinline__ void adamw_load(BlockIn& in, const AdamArgs& a, const TableEntry& t, uint64_t b, uint32_t lane, uint64_t e0, uint32_t left) {
    Raw &mr = in.mr, &vr = in.vr;
    if (WIDE && t.status && one_record(t)) in.st = record(t, (e0 + lane * 8) >> t.k_shift);
    load_raw<WIDE>(in.gr, t.grad, t.grad_dtype, e0, lane, left);
    load_raw<WIDE>(in.pr, t.master ? t.master : t.param, t.master ? (uint32_t)FTC_F32 : t.param_dtype, e0, lane, left);
    const uint64_t q = b * FTC_STATE_BLOCK;
    const uint8_t *mp = static_cast<const uint8_t*>(a.m) + q, *vp = static_cast<const uint8_t*>(a.v) + q;
    if (BITS == 32) {
        load_raw<WIDE>(mr, a.m, FTC_F32, q, lane, FTC_STATE_BLOCK);
        load_raw<WIDE>(vr, a.v, FTC_F32, q, lane, FTC_STATE_BLOCK);
    } else {
        if (WIDE) {
            const uint2 x = reinterpret_cast<const uint2*>(mp)[lane], y = reinterpret_cast<const uint2*>(vp)[lane];
            mr.r[0] = x.x; mr.r[1] = x.y; vr.r[0] = y.x; vr.r[1] = y.y;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) { mr.r[j] = mp[j * 32 + lane]; vr.r[j] = vp[j * 32 + lane]; }
        }
        in.ms = a.m_scale[b]; in.vs = a.v_scale[b];
    }
}

template <int BITS, bool WIDE, bool DITHER>
__device__ __forceinline__ void adamw_block(const BlockIn& in, const AdamArgs& a, const TableEntry& t, uint64_t b, uint32_t lane, uint64_t e0, uint32_t left, float scale) {
    const Raw &gr = in.gr, &pr = in.pr;
    Raw mr = in.mr, vr = in.vr;
    float ms = in.ms, vs = in.vs;
    const uint32_t pd = t.master ? (uint32_t)FTC_F32 : t.param_dtype;
    void* weights = t.master ? t.master : t.param;
    const uint64_t q = b * FTC_STATE_BLOCK;
    uint8_t *mp = static_cast<uint8_t*>(a.m) + q, *vp = static_cast<uint8_t*>(a.v) + q;
    F2 g[4], p[4], m[4], v[4];
    uint32_t live;
    numbers<WIDE>(g, gr, t.grad_dtype);
    if (t.status) {
        F2 w[4];
        if (WIDE && one_record(t)) {
            const float s = share_of(in.st);
            live = s > 0.f ? 0xFFu : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = twice(s);
        } else live = shares<WIDE>(w, t, e0, lane, left);
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = mul(g[i], w[i]);
    } else live = inside<WIDE>(lane, left);
    numbers<WIDE>(p, pr, pd);
    if (BITS == 32) { numbers<true>(m, mr, FTC_F32); numbers<true>(v, vr, FTC_F32); }
    else {
        const F2 mk = twice(ms * kInv127), vk = twice(vs * kInv255);
        if (WIDE) { mr.r[0] ^= 0x80808080u; mr.r[1] ^= 0x80808080u; }           // signed bytes + 128
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = i * 2 % 4;
            const F2 c = WIDE ? bytes_numbers(byte_of(mr.r[i / 2], j), byte_of(mr.r[i / 2], j + 1), twice(-8388736.f))
                              : bytes_numbers(mr.r[2 * i] ^ 0x4B000080u, mr.r[2 * i + 1] ^ 0x4B000080u, twice(-8388736.f));
            const F2 d = WIDE ? bytes_numbers(byte_of(vr.r[i / 2], j), byte_of(vr.r[i / 2], j + 1), twice(-8388608.f))
                              : bytes_numbers(vr.r[2 * i] | 0x4B000000u, vr.r[2 * i + 1] | 0x4B000000u, twice(-8388608.f));
            const F2 r = mul(mul(d, d), vk);
            m[i] = mul(pair(__fmul_rn(lo(c), fabsf(lo(c))), __fmul_rn(hi(c), fabsf(hi(c)))), mk);
            v[i] = mul(r, r);
        }
    }
    const float lr = a.lr * t.lr_scale;
    const F2 keep = twice(1.f - lr * t.weight_decay), rate = twice(-(lr * a.fix1)), sc = twice(scale);
    const bool some = t.status && live != 0xFFu;                                // messages missing
    F2 root[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = mul(g[i], sc);
        const F2 mi = add_apart(mul(m[i], twice(a.beta1)), mul(g[i], twice(a.rest1)), twice(a.one));
        const F2 vi = add_apart(mul(v[i], twice(a.beta2)), mul(mul(g[i], g[i]), twice(a.rest2)), twice(a.one));
        if (BITS == 8 && some) {                                                // the block's codes need all; in 32 bits the live are stored
            const bool x = live >> (2 * i) & 1u, y = live >> (2 * i + 1) & 1u;
            m[i] = pair(x ? lo(mi) : lo(m[i]), y ? hi(mi) : hi(m[i]));
            v[i] = pair(x ? lo(vi) : lo(v[i]), y ? hi(vi) : hi(v[i]));
        } else { m[i] = mi; v[i] = vi; }
        root[i] = BITS == 8 ? pair(fast_root(lo(v[i])), fast_root(hi(v[i]))) : pair(fast_root_of_any(lo(v[i])), fast_root_of_any(hi(v[i])));
    }
    if (BITS == 8) {                                                            // subnormal numbers among v, or zeros: the rest has done without
        float least = lo(root[0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) least = smallest(least, i ? lo(root[i]) : hi(root[0]), hi(root[i]));
        if (!(least > 0.f)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) root[i] = pair(fast_root_of_any(lo(v[i])), fast_root_of_any(hi(v[i])));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 den = add(mul(root[i], twice(a.fix2)), twice(a.eps));
        p[i] = fma(mul(m[i], pair(fast_inverse(lo(den)), fast_inverse(hi(den)))), rate, mul(p[i], keep));
    }
    store_numbers<WIDE>(weights, pd, e0, lane, p, live);
    if (t.master) store_numbers<WIDE>(t.param, t.param_dtype, e0, lane, p, live);
    if (BITS == 32) {
        store_numbers<WIDE>(a.m, FTC_F32, q, lane, m, live);
        store_numbers<WIDE>(a.v, FTC_F32, q, lane, v, live);
        return;
    }
    if (t.status && !__any_sync(0xFFFFFFFFu, live)) return;
    float mm = 0.f, vm = 0.f;                                                   // behind the tensor's end all is zero
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mm = largest(mm, lo(m[i]), hi(m[i]));
        vm = largest(vm, lo(v[i]), hi(v[i]));
    }
    ms = warp_max_bits(__float_as_uint(mm)); vs = __fsqrt_rn(warp_max_bits(__float_as_uint(vm)));     // the root keeps the order: the largest root
    ms = ms <= 3.402823466e38f ? fmaxf(ms, kTiny) : __uint_as_float(0x7FC00000u);
    vs = vs <= 3.402823466e38f ? fmaxf(vs, kTiny) : __uint_as_float(0x7FC00000u);
    const float inv = 1.f / (lane & 1 ? vs : ms);                               // one division for both
    const float mi = __shfl_sync(0xFFFFFFFFu, inv, 0), vi = __shfl_sync(0xFFFFFFFFu, inv, 1);
    F2 c[4], d[4];
    float far_m = 0.f, far_v = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 xm = mul(pair(__fmul_rn(fabsf(lo(m[i])), mi), __fmul_rn(fabsf(hi(m[i])), mi)), twice(16129.f)), xv = mul(mul(root[i], twice(vi)), twice(65025.f));
        if (DITHER) {
            const F2 u = pair(dither((uint32_t)q + at<WIDE>(lane, 2 * i), a.phase), dither((uint32_t)q + at<WIDE>(lane, 2 * i + 1), a.phase));
            c[i] = a.dither & kDitherM ? dithered_roots<false>(xm, u, 127.f) : likely_roots(xm, far_m);
            d[i] = a.dither & kDitherV ? dithered_roots<true>(xv, u, 255.f) : likely_roots(xv, far_v);
        } else {
            c[i] = likely_roots(xm, far_m);
            d[i] = likely_roots(xv, far_v);
        }
    }
    if (!(far_m < 0.5f - kDoubtM)) {                                            // one lane in three thousand, and NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = pair(nearest_root(fabsf(lo(m[i])) * mi * 16129.f, 127.f), nearest_root(fabsf(hi(m[i])) * mi * 16129.f, 127.f));
    }
    if (!(far_v < 0.5f - kDoubtV)) {                                            // one in seven hundred
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = pair(nearest_root(__fsqrt_rn(lo(v[i])) * vi * 65025.f, 255.f), nearest_root(__fsqrt_rn(hi(v[i])) * vi * 65025.f, 255.f));
    }
    float least = 255.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) least = smallest(least, lo(d[i]), hi(d[i]));
    if (!(least >= 1.f)) {                                                      // a root above zero has a code above zero
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = pair(fmaxf(lo(d[i]), one_above(lo(v[i]))), fmaxf(hi(d[i]), one_above(hi(v[i]))));
    }
    uint32_t cm[8], cv[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 s = add(pair(copysignf(lo(c[i]), lo(m[i])), copysignf(hi(c[i]), hi(m[i]))), twice(kWhole)), u = add(d[i], twice(kWhole));
        cm[2 * i] = __float_as_uint(lo(s)); cm[2 * i + 1] = __float_as_uint(hi(s));
        cv[2 * i] = __float_as_uint(lo(u)); cv[2 * i + 1] = __float_as_uint(hi(u));
    }
    if (WIDE) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t* w = i < 2 ? cm + 4 * i : cv + 4 * (i - 2);
            x[i] = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
        }
        reinterpret_cast<uint2*>(mp)[lane] = make_uint2(x[0], x[1]);
        reinterpret_cast<uint2*>(vp)[lane] = make_uint2(x[2], x[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) { mp[j * 32 + lane] = (uint8_t)cm[j]; vp[j * 32 + lane] = (uint8_t)cv[j]; }
    }
    if (lane == 0) { a.m_scale[b] = ms; a.v_scale[b] = vs; }
}

template <int BITS, bool WIDE, bool DITHER>
__device__ __forceinline__ void adamw_one(const AdamArgs& a, const TableEntry& t, uint64_t b, uint32_t lane, uint64_t e0, uint32_t left, float scale) {
    BlockIn in;
    adamw_load<BITS, WIDE>(in, a, t, b, lane, e0, left);
    adamw_block<BITS, WIDE, DITHER>(in, a, t, b, lane, e0, left, scale);
}

// A warp takes one block; 32 warps an SM, no loop: the table's entry and the block's loads are the whole wait, and other warps fill it. 32-bit
// states run at a copy's speed (101M elements, bf16 weights with a float32 copy, records: 455-470 us, 6.6 TB/s); states in 8 bits take
// 79 instructions an element the narrow way (packed odd tensors, 17M elements: 68 us, 3.6 TB/s, 61 % of the issue slots), which bounds them.
// WIDE: full blocks of aligned tensors go the wide way; else all go the narrow one.
template <int BITS, bool WIDE, bool DITHER>
__global__ void __launch_bounds__(kWarps * 32, 4) adamw_kernel(AdamArgs a) {
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t b = blockIdx.x * (uint64_t)kWarps + (threadIdx.x >> 5);
    if (b >= a.n_blocks) return;
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    const TableEntry t = table_entries(a.table)[table_map(a.table, a.n_params)[b]];
    if (!isfinite(scale)) return;
    const uint64_t e0 = (b - t.first_block) * FTC_STATE_BLOCK, left = t.n - e0;
    if (WIDE && t.wide && left >= FTC_STATE_BLOCK) adamw_one<BITS, true, DITHER>(a, t, b, lane, e0, FTC_STATE_BLOCK, scale);
    else adamw_one<BITS, false, DITHER>(a, t, b, lane, e0, left < FTC_STATE_BLOCK ? (uint32_t)left : FTC_STATE_BLOCK, scale);
}

// States in 8 bits, whose arithmetic (63 instructions an element, 74 where v is dithered) takes about as long as the memory: 201M elements in 563 to
// 635 us, 5.1 to 5.7 TB/s, 64 % of the issue slots; a quarter of them 151 us, dithered 168. Prefetch by way of shared memory at 24 or 32 warps an SM
// spilled and was slower (695, 820 us when the walk took 606). A warp takes `span` blocks one after the other, the next one's loads out while it works
// on the present one.
constexpr uint32_t kWalkWarps = 8, kWalkBlocks = 2;
template <bool DITHER> __global__ void __launch_bounds__(kWalkWarps * 32, kWalkBlocks) adamw_walk_kernel(AdamArgs a, uint64_t span) {
    const uint32_t lane = threadIdx.x & 31;
    uint64_t b = (blockIdx.x * (uint64_t)kWalkWarps + (threadIdx.x >> 5)) * span;
    const uint64_t stop = b + span < a.n_blocks ? b + span : a.n_blocks;
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!isfinite(scale)) return;
    while (b < stop) {
        const TableEntry t = table_entries(a.table)[table_map(a.table, a.n_params)[b]];
        const uint64_t last = t.first_block + (t.n + FTC_STATE_BLOCK - 1) / FTC_STATE_BLOCK, end = last < stop ? last : stop;
        const uint64_t whole = t.wide ? t.first_block + t.n / FTC_STATE_BLOCK : 0, end_wide = whole < end ? whole : end;
        uint64_t e0 = (b - t.first_block) * FTC_STATE_BLOCK;
        if (b < end_wide) {
            BlockIn next;
            adamw_load<8, true>(next, a, t, b, lane, e0, FTC_STATE_BLOCK);
            for (; b < end_wide; ++b, e0 += FTC_STATE_BLOCK) {
                const BlockIn in = next;
                if (b + 1 < end_wide) adamw_load<8, true>(next, a, t, b + 1, lane, e0 + FTC_STATE_BLOCK, FTC_STATE_BLOCK);
                adamw_block<8, true, DITHER>(in, a, t, b, lane, e0, FTC_STATE_BLOCK, scale);
            }
        }
        for (; b < end; ++b, e0 += FTC_STATE_BLOCK)
            adamw_one<8, false, DITHER>(a, t, b, lane, e0, t.n - e0 < FTC_STATE_BLOCK ? (uint32_t)(t.n - e0) : FTC_STATE_BLOCK, scale);
    }
}

cudaError_t launch_adamw(const AdamArgs& a, int sms, cudaStream_t st) {
    // The walk pays from about twelve blocks a warp on, where the tensors no longer lie in L2: blocks a warp 4, 8, 16, 29, 331: 8.8, 15.5, 28.6, 53, 563 us
    // against 8.0, 14.1, 31.0, 55, 614 a block for each warp. The narrow way has too much in registers for it (packed tensors, 4 to 29 blocks a warp:
    // 13.6 to 81 us against 11.1 to 69).
    const uint64_t warps = (uint64_t)sms * kWalkWarps * kWalkBlocks;
    if (a.bits == 8 && a.mostly_wide && a.n_blocks >= warps * 4) {
        (a.dither ? adamw_walk_kernel<true> : adamw_walk_kernel<false>)<<<sms * kWalkBlocks, kWalkWarps * 32, 0, st>>>(a, (a.n_blocks + warps - 1) / warps);
        return cudaGetLastError();
    }
    const uint32_t grid = (uint32_t)((a.n_blocks + kWarps - 1) / kWarps);
    if (a.bits == 32) {
        (a.mostly_wide ? adamw_kernel<32, true, false> : adamw_kernel<32, false, false>)<<<grid, kWarps * 32, 0, st>>>(a);
    } else if (a.dither) {
        (a.mostly_wide ? adamw_kernel<8, true, true> : adamw_kernel<8, false, true>)<<<grid, kWarps * 32, 0, st>>>(a);
    } else {
        (a.mostly_wide ? adamw_kernel<8, true, false> : adamw_kernel<8, false, false>)<<<grid, kWarps * 32, 0, st>>>(a);
    }
    return cudaGetLastError();
}

// A lane reads 8 codes of each state (8 bytes) and writes 32 bytes of each output. Bound by memory (201M elements: 300 us, 6.7 TB/s).
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

cudaError_t launch_adamw_states(uint64_t blocks, const void* m, const void* v, const float* ms, const float* vs, float* mo, float* vo, cudaStream_t st) {
    adamw_states_kernel<<<(uint32_t)((blocks + 7) / 8), 256, 0, st>>>(blocks, static_cast<const uint8_t*>(m), static_cast<const uint8_t*>(v), ms, vs, mo, vo);
    return cudaGetLastError();
}

// ---- the norm: one pass over the gradients, bound by memory where they are many (202M elements in float32 with a record for each 32:
// 156 us, 5.8 TB/s), by two kernels' beginnings where they are few. Warp w adds up the squares of the blocks [w*span, (w+1)*span) and leaves one sum for each tensor it meets; warp w and
// tensor t share slot w + t (going on by one block either grows, so no two pairs with blocks in common share a slot)

// Sum of the squares of 8 numbers. In float32 where that neither overflows nor loses small squares (4 roundings at most one after the
// other), else in float64.
__device__ __noinline__ double squares_64(F2 a, F2 b, F2 c, F2 d) {
    const F2 g[4] = {a, b, c, d};
    double s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) s += (double)lo(g[i]) * lo(g[i]) + (double)hi(g[i]) * hi(g[i]);
    return s;
}
__device__ __forceinline__ double squares(const F2* g) {
    const F2 s = add(fma(g[0], g[0], mul(g[1], g[1])), fma(g[2], g[2], mul(g[3], g[3])));
    const float f = lo(s) + hi(s);
    return f >= 1e-30f && f <= 1e38f ? (double)f : squares_64(g[0], g[1], g[2], g[3]);
}

// Elements e .. end - 1 of any tensor, two pieces of 256 under way.
__device__ __forceinline__ double piece_squares(const Raw& x, const TableEntry& t, uint64_t e, uint32_t left) {
    F2 g[4];
    numbers<false>(g, x, t.grad_dtype);
    if (t.status) {
        F2 w[4];
        const uint32_t live = shares<false>(w, t, e, threadIdx.x & 31, left);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            g[i] = mul(g[i], w[i]);
            g[i] = pair(live >> (2 * i) & 1u ? lo(g[i]) : 0.f, live >> (2 * i + 1) & 1u ? hi(g[i]) : 0.f);
        }
    }
    return squares(g);                                               // elements behind the end were loaded as zeros
}
__device__ __forceinline__ double walk_squares(const TableEntry& t, uint64_t e, uint64_t end) {
    const uint32_t lane = threadIdx.x & 31;
    double s = 0;
    for (; e < end; e += 2 * FTC_STATE_BLOCK) {
        Raw x, y;
        const uint64_t rest = end - e;
        const uint32_t left = rest < FTC_STATE_BLOCK ? (uint32_t)rest : FTC_STATE_BLOCK;
        const uint32_t more = rest <= FTC_STATE_BLOCK ? 0 : rest < 2 * FTC_STATE_BLOCK ? (uint32_t)rest - FTC_STATE_BLOCK : FTC_STATE_BLOCK;
        load_raw<false>(x, t.grad, t.grad_dtype, e, lane, left);
        if (more) load_raw<false>(y, t.grad, t.grad_dtype, e + FTC_STATE_BLOCK, lane, more);
        s += piece_squares(x, t, e, left);
        if (more) s += piece_squares(y, t, e + FTC_STATE_BLOCK, more);
    }
    return s;
}

// `pieces` times 256 elements of one type; this lane's first eight are e .. e + 7, on a boundary of eight. A lane's eight have
// no record, one (the records of neighbouring pieces lie a fixed way apart then), or up to two or three (82M elements in float32 with a
// record for each 7: 104 us; element by element by way of the warp's lanes 262).
template <uint32_t DTYPE, int RECORDS, bool SOLO> __device__ __forceinline__ double run_squares(const TableEntry& t, uint64_t e, uint32_t pieces) {
    constexpr uint32_t BYTES = FTC_STATE_BLOCK * (DTYPE == FTC_F32 ? 4 : 2), RECORD = FTC_STATUS_WORDS / 2;
    constexpr int AHEAD = SOLO ? RECORDS >= 2 ? 2 : 4 : DTYPE == FTC_F32 || RECORDS >= 2 ? 4 : 8;       // pieces whose loads are out at once: 4 KB a warp; fewer in the lone block's 64 registers
    struct In { Raw x; uint2 a, b, c; uint32_t split; };                // a: for the first `split` elements, b: for the k after them
    const char* p = static_cast<const char*>(t.grad) + e * (BYTES / FTC_STATE_BLOCK);
    const uint2* st = nullptr;
    uint64_t next = 0;
    uint32_t place = 0, over = 0, k = 0;
    if (RECORDS) {
        k = t.k;
        st = reinterpret_cast<const uint2*>(t.status) + message_of(t, e, place) * RECORD;
        next = (uint64_t)(FTC_STATE_BLOCK / k) * RECORD;
        over = FTC_STATE_BLOCK % k;
    }
    const auto load = [&](In& in, int i) {                           // of the piece i from here
        if (RECORDS) in.a = st[i * next];
        if (RECORDS >= 2) {
            in.split = k - place;
            in.b = st[in.split < 8 ? RECORD : 0];
        }
        if (RECORDS == 3) in.c = st[in.split + k < 8 ? 2 * RECORD : 0];
        if (DTYPE == FTC_F32) load_32(p + i * BYTES, in.x.r);
        else load_16(p + i * BYTES, in.x.r);
    };
    const auto go_on = [&](int i) {                                  // i pieces; one at a time where a place in the message is kept
        p += i * BYTES;
        if (RECORDS) st += i * next;
        if (RECORDS >= 2) {
            place += over;
            if (place >= k) { place -= k; st += RECORD; }
        }
    };
    constexpr bool EACH = RECORDS >= 2;
    double s = 0;
    const auto add_one = [&](const In& in) {
        F2 g[4];
        numbers<true>(g, in.x, DTYPE);
        const float a = RECORDS ? share_of(in.a) : 1.f;
        if (RECORDS >= 2) {
            const float b = share_of(in.b), c = RECORDS == 3 ? share_of(in.c) : 0.f;
            const auto shared = [&](float x, uint32_t j) {
                const float f = j < in.split ? a : RECORDS == 2 || j < in.split + k ? b : c;
                return f > 0.f ? x * f : 0.f;                        // what was not delivered may be NaN
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = pair(shared(lo(g[i]), 2 * i), shared(hi(g[i]), 2 * i + 1));
            s += squares(g);
        } else if (a > 0.f) s = ::fma((double)a * a, squares(g), s);
    };
    for (; pieces >= AHEAD; pieces -= AHEAD) {
        In in[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) { load(in[i], EACH ? 0 : i); if (EACH) go_on(1); }
        if (!EACH) go_on(AHEAD);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) add_one(in[i]);
    }
    if (pieces) {
        In in[AHEAD - 1];
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i) {                       // behind the end the last one again, not added
            const bool more = i + 1 < (int)pieces;
            load(in[i], EACH ? 0 : i < (int)pieces ? i : (int)pieces - 1);
            if (EACH && more) go_on(1);
        }
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i)
            if (i < (int)pieces) add_one(in[i]);
    }
    return s;
}
template <int RECORDS, bool SOLO> __device__ __forceinline__ double run_squares(const TableEntry& t, uint64_t e, uint32_t pieces) {
    return t.grad_dtype == FTC_F32 ? run_squares<FTC_F32, RECORDS, SOLO>(t, e, pieces)
         : t.grad_dtype == FTC_BF16 ? run_squares<FTC_BF16, RECORDS, SOLO>(t, e, pieces) : run_squares<FTC_F16, RECORDS, SOLO>(t, e, pieces);
}

// The sums of the warp w, whose first block is of tensor `ti`. Where a tensor does not begin on a boundary of 8 elements its blocks are
// taken `h` elements later, on the first such boundary; the tensor's first warp has the h elements before it, its last warp up to a block less
// (72M bf16 elements packed without padding: 44 us, with loads of single elements 55). MIXED: with the code for two and three records; without
// it the kernel is smaller and takes 156 us for 202M elements in place of 158.
template <bool SOLO, bool MIXED> __device__ __forceinline__ void warp_squares(const TableEntry* entries, uint32_t ti, uint64_t n_blocks, uint64_t span, uint64_t w, double* slots) {
    const uint32_t lane = threadIdx.x & 31;
    uint64_t b = w * span;
    const uint64_t b1 = b + span < n_blocks ? b + span : n_blocks;
    for (; b < b1; ++ti) {
        const TableEntry& t = entries[ti];
        const uint64_t n = t.n;
        if (n == 0) continue;
        const uint64_t first = t.first_block, last = first + (n + FTC_STATE_BLOCK - 1) / FTC_STATE_BLOCK, end = last < b1 ? last : b1;
        const uint32_t h = (uint32_t)(0 - reinterpret_cast<uintptr_t>(t.grad) / (t.grad_dtype == FTC_F32 ? 4 : 2)) & 7u, k = t.k;
        uint64_t e = b == first ? 0 : (b - first) * FTC_STATE_BLOCK + h, to = end == last ? n : (end - first) * FTC_STATE_BLOCK + h;
        b = end;
        if (to > n) to = n;
        double s = 0;
        if (e == 0 && h) { e = h < to ? h : to; s = walk_squares(t, 0, e); }
        if (to >= e + FTC_STATE_BLOCK) {
            const uint64_t mine = e + lane * 8;
            const uint32_t pieces = (uint32_t)((to - e) / FTC_STATE_BLOCK);
            bool run = true;
            if (!t.status) s += run_squares<0, SOLO>(t, mine, pieces);
            else if (h == 0 && k % 8 == 0 && FTC_STATE_BLOCK % k == 0) s += run_squares<1, SOLO>(t, mine, pieces);
            else if (MIXED && (k >= 7 || (k == 4 && h % 4 == 0))) s += run_squares<2, SOLO>(t, mine, pieces);          // eight neighbours meet two messages at most
            else if (MIXED && k >= 4) s += run_squares<3, SOLO>(t, mine, pieces);
            else run = false;
            if (run) e += (uint64_t)pieces * FTC_STATE_BLOCK;
        }
        if (e < to) s += walk_squares(t, e, to);
        s = warp_sum(s);
        if (lane == 0) slots[w + ti] = s;
    }
}

template <bool MIXED> __global__ void __launch_bounds__(kWarps * 32, 3) grad_squares_kernel(const void* table, uint32_t n_params, uint64_t n_blocks, uint64_t span, double* slots, uint32_t* ticket) {
    later_kernel_may_start();
    const uint64_t w = blockIdx.x * (uint64_t)kWarps + (threadIdx.x >> 5);
    if (w == 0 && (threadIdx.x & 31) == 0) *ticket = 0;
    if (w * span < n_blocks) warp_squares<false, MIXED>(table_entries(table), table_map(table, n_params)[w * span], n_blocks, span, w, slots);
}

__device__ __forceinline__ void give_norm(double s, float max_norm, float* norm) {
    const float r = (float)sqrt(s);
    norm[0] = r;
    norm[1] = !isfinite(r) ? __uint_as_float(0x7FC00000u) : r > max_norm ? max_norm / r : 1.f;
}

// Tables of few blocks and tensors: all in one thread block, entries and sums in shared memory. One against two kernels by way of the workspace, us on the
// GPU, 6 tensors in float32 of 64, 132, 160, 320, 640 blocks: 4.1, 5.1, 5.3, 6.1, 7.5 against 5.8, 6.0, 5.8, 5.8, 5.6; with records of 32
// elements 4.6, 6.2, 6.5, 7.9, 10.3 against 6.2, 5.4, 6.3, 5.9, 6.4. A call among others takes 6.2 us up to about 130 blocks, 8.2 with unaligned tensors or more.
constexpr uint32_t kSoloWarps = 32, kSoloBlocks = 160, kSoloTensors = 16;
template <bool MIXED> __global__ void __launch_bounds__(kSoloWarps * 32) grad_norm_solo_kernel(const void* table, uint32_t n_params, uint64_t n_blocks, uint64_t span, float max_norm,
                                                                         float* norm, float* norms) {
    __shared__ TableEntry entries[kSoloTensors];
    __shared__ double slots[kSoloWarps + kSoloTensors], part[kSoloWarps];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t ti = warp * span < n_blocks ? table_map(table, n_params)[warp * span] : 0;
    if (threadIdx.x < n_params * (sizeof(TableEntry) / 4))
        reinterpret_cast<uint32_t*>(entries)[threadIdx.x] = reinterpret_cast<const uint32_t*>(table_entries(table))[threadIdx.x];
    __syncthreads();
    warp_squares<true, MIXED>(entries, ti, n_blocks, span, warp, slots);
    __syncthreads();
    double all = 0;
    if (warp < n_params) {
        const uint64_t n = entries[warp].n, first = entries[warp].first_block;
        const uint32_t w0 = (uint32_t)(first / span), w1 = n ? (uint32_t)((first + (n - 1) / FTC_STATE_BLOCK) / span) + 1 : w0;      // at most kSoloWarps warps
        all = warp_sum(w0 + lane < w1 ? slots[w0 + lane + warp] : 0.0);
        if (lane == 0 && norms) norms[warp] = (float)sqrt(all);
    }
    if (lane == 0) part[warp] = all;
    __syncthreads();
    if (warp) return;
    all = warp_sum(part[lane]);
    if (lane == 0) give_norm(all, max_norm, norm);
}

__device__ __forceinline__ double block_sum(double s, double* part) {          // 128 threads
    s = warp_sum(s);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = (part[0] + part[1]) + (part[2] + part[3]);
    __syncthreads();
    return s;
}

// A block adds the slots of one tensor after the other; the block that is last to finish adds the tensors' sums. Every sum has an order of
// its own that does not depend on which block comes last.
__global__ void __launch_bounds__(128) grad_norm_kernel(const void* table, uint32_t n_params, uint64_t span, float max_norm, const double* slots, double* sums,
                                                        uint32_t* ticket, float* norm, float* norms) {
    __shared__ double part[4];
    __shared__ bool mine;
    for (uint32_t ti = blockIdx.x; ti < n_params; ti += gridDim.x) {
        const uint64_t n = table_entries(table)[ti].n, first = table_entries(table)[ti].first_block;
        double s = 0;
        wait_for_earlier_kernel();
        if (n) {
            const uint64_t last = (first + (n - 1) / FTC_STATE_BLOCK) / span;
#pragma unroll 8
            for (uint64_t w = first / span + threadIdx.x; w <= last; w += 128) s += slots[w + ti];
        }
        s = block_sum(s, part);
        if (threadIdx.x == 0) { sums[ti] = s; if (norms) norms[ti] = (float)sqrt(s); }
    }
    if (threadIdx.x == 0) {
        __threadfence();                                             // this block's sums before its ticket
        mine = atomicAdd(ticket, 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!mine) return;
    double s = 0;
    for (uint32_t ti = threadIdx.x; ti < n_params; ti += 128) s += __ldcg(sums + ti);
    s = block_sum(s, part);
    if (threadIdx.x == 0) give_norm(s, max_norm, norm);
}

// Warps that share the blocks: those that the GPU holds at once; of more than 32 blocks for each, four times as many, so that who is done
// early takes the next (202M elements: 163 us against 173).
uint32_t grad_norm_warps(uint64_t n_blocks, int sm_count) {
    const uint64_t held = (uint64_t)sm_count * kWarps * 3;
    return (uint32_t)(n_blocks < held ? n_blocks : n_blocks <= 32 * held ? held : 4 * held);
}

cudaError_t launch_grad_norm(const void* table, uint32_t n_params, uint64_t n_blocks, bool mixed, float max_norm, float* norm, float* norms, double* ws, int sm_count,
                             cudaStream_t st) {
    const bool solo = n_blocks <= kSoloBlocks && n_params <= kSoloTensors;
    const uint32_t warps = solo ? kSoloWarps : grad_norm_warps(n_blocks, sm_count);
    const uint64_t span = n_blocks ? (n_blocks + warps - 1) / warps : 1;
    double *slots = ws + 1, *sums = slots + warps + n_params;
    uint32_t* ticket = reinterpret_cast<uint32_t*>(ws);
    if (solo) {
        (mixed ? grad_norm_solo_kernel<true> : grad_norm_solo_kernel<false>)<<<1, kSoloWarps * 32, 0, st>>>(table, n_params, n_blocks, span, max_norm, norm, norms);
        return cudaGetLastError();
    }
    (mixed ? grad_squares_kernel<true> : grad_squares_kernel<false>)<<<warps ? (warps + kWarps - 1) / kWarps : 1, kWarps * 32, 0, st>>>(table, n_params, n_blocks, span, slots, ticket);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const uint32_t cap = (uint32_t)sm_count * 8;
    return launch_second(grad_norm_kernel, n_params < cap ? n_params : cap, 128, st, table, n_params, span, max_norm, (const double*)slots, sums, ticket, norm, norms);
}

}  // namespace ftc
