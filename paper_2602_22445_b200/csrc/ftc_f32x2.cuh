// Pairs of float32 numbers in one 64-bit register, for the packed instructions (each half rounded as the plain one is).
#pragma once
#include <cstdint>

namespace ftc {

struct F2 { unsigned long long v; };

__device__ __forceinline__ F2 pair(float lo, float hi) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ F2 twice(float x) { return pair(x, x); }
__device__ __forceinline__ float lo(F2 a) { float x; asm("{ .reg .f32 t; mov.b64 {%0, t}, %1; }" : "=f"(x) : "l"(a.v)); return x; }
__device__ __forceinline__ float hi(F2 a) { float x; asm("{ .reg .f32 t; mov.b64 {t, %0}, %1; }" : "=f"(x) : "l"(a.v)); return x; }
__device__ __forceinline__ F2 add(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 mul(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }

// The sum of two products that were rounded before. The assembler joins a packed product and a packed sum into one multiply-add, so the
// sum is a multiply-add itself, with a factor of 1 (twice) that only the host knows.
__device__ __forceinline__ F2 add_apart(F2 a, F2 b, F2 one) { return fma(a, one, b); }

}  // namespace ftc
