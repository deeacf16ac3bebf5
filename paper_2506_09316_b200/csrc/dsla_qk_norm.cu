// Norm of each head of queries and keys and the rotation by the token's position, one pass: rows of a projection in, rows of q and k out.
//     y = w x r,   r = rsqrt(mean(x^2) + eps) | rsqrt(sum(x^2) + eps) | 1;      (a, b) -> (a cos f - b sin f, b cos f + a sin f)
// A lane holds two pieces of four channels of a head, chosen so that the channels that turn with each other are its own: i and i + rot/2 (or the
// neighbours 2i, 2i + 1), so only the sum of squares crosses lanes (with eight neighbouring channels to a lane the rotation took eight shuffles, and
// the shuffles the time: 37 us for 4096 tokens of 64 heads of 128 in bf16, now 28, 4.8 TB/s; fetching rounds ahead through shared memory, or several tokens a CTA, made it no
// shorter).  A CTA takes the heads of one token: the rot/2 angles and their sines are computed once for all of them, while the
// first heads are on their way.  An angle is a product in fp64, reduced to half turns there: at position 100,000 an fp32 product is off by
// 4e-3 radians.  Bound by HBM: x read once, y written once.
#include "dsla_internal.cuh"

namespace dsla {

namespace {

constexpr int QN_THREADS = 256;

// Four neighbouring channels.
template <typename T> struct Four;
template <> struct Four<float> {
    float4 a;
    __device__ __forceinline__ void zero() { a = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void get(float* x) const { x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; }
    static __device__ __forceinline__ void store(float* p, const float* x) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct Four<__nv_bfloat16> {
    uint2 a;
    __device__ __forceinline__ void zero() { a = make_uint2(0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void get(float* x) const {
        x[0] = __uint_as_float(a.x << 16); x[1] = __uint_as_float(a.x & 0xffff0000u);
        x[2] = __uint_as_float(a.y << 16); x[3] = __uint_as_float(a.y & 0xffff0000u);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* x) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(x[0], x[1]), hi = __floats2bfloat162_rn(x[2], x[3]);
        *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
};

template <int D, typename T, int NORM, bool INTERLEAVED>
__global__ void __launch_bounds__(QN_THREADS) qk_norm_rope_kernel(const dsla_qk_norm_rope_args p) {
    constexpr int LANES = D / 8, HEADS = QN_THREADS / LANES;      // lanes per head, heads per CTA at a time
    constexpr int AHEAD = 4;                                      // rounds of heads whose loads are issued together
    __shared__ __align__(16) float scos[D / 2], ssin[D / 2];
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
    float wq[8], wk[8], cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = (i < 4 ? at0 : at1) + (i & 3);
        wq[i] = p.q_weight ? __ldg(p.q_weight + at) : 1.f;
        wk[i] = p.k_weight ? __ldg(p.k_weight + at) : 1.f;
    }
    if (rot > 0) {
        if (tid < half) {
            const double turned = (double)p.positions[t] * (double)p.inv_freq[tid] * 0.31830988618379067154;      // half turns
            sincospif((float)(turned - 2.0 * rint(0.5 * turned)), &ssin[tid], &scos[tid]);
        }
        __syncthreads();
        if (turns) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { cs[i] = scos[4 * lane + i]; sn[i] = ssin[4 * lane + i]; }
        }
    }
    for (int h0 = 0; h0 < end; h0 += AHEAD * HEADS) {
        if (h0 > 0) load(h0);
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            if (h0 + r * HEADS >= end) break;
            const int h = h0 + r * HEADS + tid / LANES;      // heads behind the last: zeros, not stored; the shuffles run in all lanes
            const bool is_k = h >= p.H;
            float x[8];
            in[r][0].get(x);
            in[r][1].get(x + 4);
            if (NORM != DSLA_NORM_NONE) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
                for (int m = 1; m < LANES; m <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
                const float f = rsqrtf((NORM == DSLA_NORM_RMS ? sum * (1.f / D) : sum) + p.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= is_k ? wk[i] : wq[i];
            if (turns) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int a = INTERLEAVED ? 2 * i : i, b = INTERLEAVED ? 2 * i + 1 : i + 4;
                    const float u = x[a], v = x[b];
                    x[a] = fmaf(u, cs[i], -(v * sn[i]));
                    x[b] = fmaf(v, cs[i], u * sn[i]);
                }
            }
            if (h < end) {
                T* dst = is_k ? reinterpret_cast<T*>(p.k_out) + (size_t)t * p.k_out_stride + (size_t)(h - p.H) * D
                              : reinterpret_cast<T*>(p.q_out) + (size_t)t * p.q_out_stride + (size_t)h * D;
                Four<T>::store(dst + at0, x);
                Four<T>::store(dst + at1, x + 4);
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
