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
// ROUNDED: the high term is; cut off, it leaves a low term of x's own sign, which the MMA cuts off towards zero again (2^-22 that always go one way).
template <bool ROUNDED>
__device__ __forceinline__ void tf32_terms(float x, uint32_t& hi, uint32_t& lo) {
    hi = (__float_as_uint(x) + (ROUNDED ? 0x1000u : 0u)) & 0xffffe000u;
    lo = __float_as_uint(x - __uint_as_float(hi));
}
// c[n] = M[16 x 8 KT] B_n[8 KT x 8], all in shared memory: element (m, k) of M at m * mr + k * mk, (k, i) of B_n at n * bt + k * bk + i * bn; steps of 8 from k_first up to
// k_last - 1.  Thread (r, q) = (lane / 4, lane % 4) has rows r, r + 8 and columns 2 q, 2 q + 1: c[n][0], c[n][1] and c[n][2], c[n][3].
template <int KT, int NT, bool ROUNDED>
__device__ __forceinline__ void products(float (&c)[NT][4], const float* M, int mr, int mk, const float* B, int bk, int bn, int bt, int k_first, int k_last, int lane) {
    const int r = lane >> 2, q = lane & 3;
    float c1[NT][4] = {}, c2[NT][4] = {};      // (three sums side by side: an MMA waits 35 cycles for the one before it)
#pragma unroll
    for (int n = 0; n < NT; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
#pragma unroll
    for (int k = 0; k < KT; ++k) {
        if (k < k_first || k >= k_last) continue;
        uint32_t ah[4], al[4], bh[NT][2], bl[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) tf32_terms<ROUNDED>(B[n * bt + (8 * k + q + 4 * i) * bk + r * bn], bh[n][i], bl[n][i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) tf32_terms<ROUNDED>(M[(r + 8 * (i & 1)) * mr + (8 * k + q + 4 * (i >> 1)) * mk], ah[i], al[i]);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            mma_tf32(c1[n], al, bh[n]);
            mma_tf32(c2[n], ah, bl[n]);
            mma_tf32(c[n], ah, bh[n]);
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[n][i] += c1[n][i] + c2[n][i];
}
template <int KT>
__device__ __forceinline__ void product(float (&c)[4], const float* M, int mr, int mk, const float* B, int bk, int bn, int k_first, int k_last, int lane) {
    float x[1][4];
    products<KT, 1, true>(x, M, mr, mk, B, bk, bn, 0, k_first, k_last, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = x[0][i];
}
// A 16 x 8 fragment to a matrix of pitch `pitch`, scaled.
__device__ __forceinline__ void put_fragment(float* M, int pitch, const float (&c)[4], float f, int lane) {
    const int r = lane >> 2, q = lane & 3;
    *reinterpret_cast<float2*>(M + r * pitch + 2 * q) = make_float2(f * c[0], f * c[1]);
    *reinterpret_cast<float2*>(M + (r + 8) * pitch + 2 * q) = make_float2(f * c[2], f * c[3]);
}

}  // namespace dsla
