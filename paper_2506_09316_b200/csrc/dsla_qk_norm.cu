// Norm of each head of queries and keys and the rotation by the token's position, one pass: rows of a projection in, rows of q and k out.
//     y = w x r,   r = rsqrt(mean(x^2) + eps) | rsqrt(sum(x^2) + eps) | 1;      (a, b) -> (a cos f - b sin f, b cos f + a sin f)
// A lane holds two pieces of four channels of a head, chosen so that the channels that turn with each other are its own: i and i + rot/2 (or the
// neighbours 2i, 2i + 1), so only the sum of squares crosses lanes (with eight neighbouring channels to a lane the rotation took eight shuffles, and
// the shuffles the time: 37 us for 4096 tokens of 64 heads of 128 in bf16, now 27; fetching rounds ahead through shared memory, several tokens a CTA, or more CTAs an SM
// made it no shorter).  A CTA takes the heads of one token: the rot/2 angles and their sines are computed once for all of them, while the
// first heads are on their way.  An angle is a product in fp64, reduced to half turns there: at position 100,000 an fp32 product is off by
// 4e-3 radians.  x is read once, y written once.  Bound by HBM and, on top of it, the instructions (issue slots 65 % busy): the same loads and stores without norm, weights and rotation take 21.8 of the 27.1 us (6.2 TB/s),
// without the norm 24.3, without the rotation 25.1.
#include "dsla_delta.cuh"

namespace dsla {

namespace {

constexpr int QN_THREADS = 256;

// A lane's eight channels as pairs of fp32: u the first of those that turn with each other, v the second.  They come from two pieces of four
// neighbours: piece 0 and 1, or, interleaved, the even and the odd channels of both.
struct Eight { uint64_t u[2], v[2]; };
template <typename T> struct Four;
template <> struct Four<float> {
    float4 a;
    __device__ __forceinline__ void zero() { a = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ uint64_t first() const { return pair(a.x, a.y); }
    __device__ __forceinline__ uint64_t second() const { return pair(a.z, a.w); }
    __device__ __forceinline__ uint64_t even() const { return pair(a.x, a.z); }
    __device__ __forceinline__ uint64_t odd() const { return pair(a.y, a.w); }
    static __device__ __forceinline__ void store(float* p, float x, float y, float z, float w) { *reinterpret_cast<float4*>(p) = make_float4(x, y, z, w); }
};
template <> struct Four<__nv_bfloat16> {
    uint2 a;
    __device__ __forceinline__ void zero() { a = make_uint2(0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ uint64_t first() const { return pair(a.x << 16, a.x & 0xffff0000u); }
    __device__ __forceinline__ uint64_t second() const { return pair(a.y << 16, a.y & 0xffff0000u); }
    __device__ __forceinline__ uint64_t even() const { return pair(a.x << 16, a.y << 16); }
    __device__ __forceinline__ uint64_t odd() const { return pair(a.x & 0xffff0000u, a.y & 0xffff0000u); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, float x, float y, float z, float w) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(x, y), hi = __floats2bfloat162_rn(z, w);
        *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
};

template <int D, typename T, int NORM, bool INTERLEAVED>
__global__ void __launch_bounds__(QN_THREADS) qk_norm_rope_kernel(const dsla_qk_norm_rope_args p) {
    constexpr int LANES = D / 8, HEADS = QN_THREADS / LANES;      // lanes per head, heads per CTA at a time
    constexpr int AHEAD = 4;                                      // rounds of heads whose loads are issued together
    __shared__ __align__(16) float scos[D / 2], ssin[D / 2];
    __shared__ float4 weight[2][2][LANES];                        // of q and k: u's and v's of each lane
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid % LANES;
    const int rot = p.rot, half = rot / 2;
    const bool turns = lane < rot / 8;                            // this lane's channels turn
    const int at0 = !INTERLEAVED && turns ? 4 * lane : 8 * lane, at1 = !INTERLEAVED && turns ? half + 4 * lane : 8 * lane + 4;
    const int end = p.H + p.H_k;                                  // heads, q's first
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Four<T> in[AHEAD][2];
    auto load = [&](int h0) {
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            const int h = h0 + r * HEADS + tid / LANES;
            if (h < end) {
                const T* src = h >= p.H ? reinterpret_cast<const T*>(p.k) + (size_t)t * p.k_stride + (size_t)(h - p.H) * D
                                        : reinterpret_cast<const T*>(p.q) + (size_t)t * p.q_stride + (size_t)h * D;
                in[r][0].load(src + at0);
                in[r][1].load(src + at1);
            } else {
                in[r][0].zero();
                in[r][1].zero();
            }
        }
    };
    load(0);
    if (tid < 4 * LANES) {
        const int of = tid / (2 * LANES), part = tid / LANES & 1;
        const float* w = of ? p.k_weight : p.q_weight;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = INTERLEAVED ? 8 * lane + 2 * i + part : (part ? at1 : at0) + i;
            x[i] = w ? __ldg(w + at) : 1.f;
        }
        weight[of][part][lane] = make_float4(x[0], x[1], x[2], x[3]);
    }
    if (tid < half) {
        const double turned = (double)p.positions[t] * (double)p.inv_freq[tid] * 0.31830988618379067154;      // half turns
        sincospif((float)(turned - 2.0 * rint(0.5 * turned)), &ssin[tid], &scos[tid]);
    }
    __syncthreads();
    uint64_t cs[2] = {0, 0}, sn[2] = {0, 0}, minus[2] = {0, 0};
    if (turns) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float2 c = *reinterpret_cast<const float2*>(scos + 4 * lane + 2 * i), s = *reinterpret_cast<const float2*>(ssin + 4 * lane + 2 * i);
            cs[i] = pair(c.x, c.y);
            sn[i] = pair(s.x, s.y);
            minus[i] = pair(-s.x, -s.y);
        }
    }
    for (int h0 = 0; h0 < end; h0 += AHEAD * HEADS) {
        if (h0 > 0) load(h0);
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            if (h0 + r * HEADS >= end) break;
            const int h = h0 + r * HEADS + tid / LANES;      // heads behind the last: zeros, not stored; the shuffles run in all lanes
            const bool is_k = h >= p.H;
            const Four<T>&c0 = in[r][0], &c1 = in[r][1];
            Eight x;
            if (INTERLEAVED) x = {{c0.even(), c1.even()}, {c0.odd(), c1.odd()}};
            else x = {{c0.first(), c0.second()}, {c1.first(), c1.second()}};
            const float4 wu = weight[is_k][0][lane], wv = weight[is_k][1][lane];
            if (NORM != DSLA_NORM_NONE) {
                const float2 s = unpair(add2(fma2(x.u[0], x.u[0], mul2(x.u[1], x.u[1])), fma2(x.v[0], x.v[0], mul2(x.v[1], x.v[1]))));
                float sum = s.x + s.y;
#pragma unroll
                for (int m = 1; m < LANES; m <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
                const float f = rsqrtf((NORM == DSLA_NORM_RMS ? sum * (1.f / D) : sum) + p.eps);
                const uint64_t ff = pair(f, f);
#pragma unroll
                for (int i = 0; i < 2; ++i) { x.u[i] = mul2(x.u[i], ff); x.v[i] = mul2(x.v[i], ff); }
            }
            x.u[0] = mul2(x.u[0], pair(wu.x, wu.y));
            x.u[1] = mul2(x.u[1], pair(wu.z, wu.w));
            x.v[0] = mul2(x.v[0], pair(wv.x, wv.y));
            x.v[1] = mul2(x.v[1], pair(wv.z, wv.w));
            if (turns) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint64_t u = x.u[i], v = x.v[i];
                    x.u[i] = fma2(u, cs[i], mul2(v, minus[i]));
                    x.v[i] = fma2(v, cs[i], mul2(u, sn[i]));
                }
            }
            if (h < end) {
                T* dst = is_k ? reinterpret_cast<T*>(p.k_out) + (size_t)t * p.k_out_stride + (size_t)(h - p.H) * D
                              : reinterpret_cast<T*>(p.q_out) + (size_t)t * p.q_out_stride + (size_t)h * D;
                const float2 u0 = unpair(x.u[0]), u1 = unpair(x.u[1]), v0 = unpair(x.v[0]), v1 = unpair(x.v[1]);
                if (INTERLEAVED) {
                    Four<T>::store(dst + at0, u0.x, v0.x, u0.y, v0.y);
                    Four<T>::store(dst + at1, u1.x, v1.x, u1.y, v1.y);
                } else {
                    Four<T>::store(dst + at0, u0.x, u0.y, u1.x, u1.y);
                    Four<T>::store(dst + at1, v0.x, v0.y, v1.x, v1.y);
                }
            }
        }
    }
}

template <int D, typename T, int NORM>
cudaError_t launch_order(const cudaLaunchConfig_t* cfg, const dsla_qk_norm_rope_args& a) {
    return a.interleaved ? cudaLaunchKernelEx(cfg, qk_norm_rope_kernel<D, T, NORM, true>, a)
                         : cudaLaunchKernelEx(cfg, qk_norm_rope_kernel<D, T, NORM, false>, a);
}
template <int D, typename T>
cudaError_t launch_norm(const cudaLaunchConfig_t* cfg, const dsla_qk_norm_rope_args& a) {
    switch (a.norm) {
        case DSLA_NORM_RMS: return launch_order<D, T, DSLA_NORM_RMS>(cfg, a);
        case DSLA_NORM_L2: return launch_order<D, T, DSLA_NORM_L2>(cfg, a);
        default: return launch_order<D, T, DSLA_NORM_NONE>(cfg, a);
    }
}

}  // namespace

dsla_status launch_qk_norm_rope(const dsla_qk_norm_rope_args* a, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a->T);
    cfg.blockDim = dim3(QN_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t rc;
    if (a->d == 128) rc = a->dtype == DSLA_BF16 ? launch_norm<128, __nv_bfloat16>(&cfg, *a) : launch_norm<128, float>(&cfg, *a);
    else rc = a->dtype == DSLA_BF16 ? launch_norm<64, __nv_bfloat16>(&cfg, *a) : launch_norm<64, float>(&cfg, *a);
    if (rc != cudaSuccess) return DSLA_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? DSLA_OK : DSLA_ERR_CUDA;
}

}  // namespace dsla
