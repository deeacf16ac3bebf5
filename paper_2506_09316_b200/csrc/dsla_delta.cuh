// Pieces shared by the kernels of the gated delta rule.
#pragma once
#include "dsla_internal.cuh"

namespace dsla {

// Pairs of fp32: one instruction for two.
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ uint64_t pair(uint32_t x, uint32_t y) { return pair(__uint_as_float(x), __uint_as_float(y)); }
__device__ __forceinline__ float2 unpair(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}

// Products of fp32 matrices on the tensor cores: each factor in two TF32 terms (22 bits), the product of the low ones left out (2^-22).
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void tf32_terms(float x, uint32_t& hi, uint32_t& lo) {
    hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;      // rounded: cut off, it would leave a low term of x's own sign, which the MMA cuts off towards zero again
    lo = __float_as_uint(x - __uint_as_float(hi));
}
// c = M[16 x 8 KT] B[8 KT x 8], both in shared memory: element (m, k) of M at m * mr + k * mk, (k, n) of B at k * bk + n * bn; steps of 8 from k_first up to
// k_last - 1.  Thread (r, q) = (lane / 4, lane % 4) has rows r, r + 8 and columns 2 q, 2 q + 1: c[0], c[1] and c[2], c[3].
template <int KT>
__device__ __forceinline__ void product(float (&c)[4], const float* M, int mr, int mk, const float* B, int bk, int bn, int k_first, int k_last, int lane) {
    const int r = lane >> 2, q = lane & 3;
    float c1[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};      // (three sums side by side: an MMA waits 35 cycles for the one before it)
    c[0] = c[1] = c[2] = c[3] = 0.f;
#pragma unroll
    for (int k = 0; k < KT; ++k) {
        if (k < k_first || k >= k_last) continue;
        uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) tf32_terms(B[(8 * k + q + 4 * i) * bk + r * bn], bh[i], bl[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) tf32_terms(M[(r + 8 * (i & 1)) * mr + (8 * k + q + 4 * (i >> 1)) * mk], ah[i], al[i]);
        mma_tf32(c1, al, bh);
        mma_tf32(c2, ah, bl);
        mma_tf32(c, ah, bh);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] += c1[i] + c2[i];
}
// A 16 x 8 fragment to a matrix of pitch `pitch`, scaled.
__device__ __forceinline__ void put_fragment(float* M, int pitch, const float (&c)[4], float f, int lane) {
    const int r = lane >> 2, q = lane & 3;
    *reinterpret_cast<float2*>(M + r * pitch + 2 * q) = make_float2(f * c[0], f * c[1]);
    *reinterpret_cast<float2*>(M + (r + 8) * pitch + 2 * q) = make_float2(f * c[2], f * c[3]);
}

}  // namespace dsla
