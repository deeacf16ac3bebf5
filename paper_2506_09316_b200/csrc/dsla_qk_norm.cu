// Norm of each head of queries and keys and the rotation by the token's position, one pass: rows of a projection in, rows of q and k out.
//     y = w x r,   r = rsqrt(mean(x^2) + eps) | rsqrt(sum(x^2) + eps) | 1;      (a, b) -> (a cos f - b sin f, b cos f + a sin f)
// A head's channels lie eight to a lane, 16-byte loads and stores; the sum of squares closes with shuffles, and so does the rotation
// in halves (channel i meets channel i + rot/2, rot/16 lanes away).  A CTA takes the heads of one token, so the rot/2 angles and their
// sines are computed once for all of them.  An angle is a product in fp64, reduced to half turns there: at position 100,000 an fp32 product is off by
// 4e-3 radians.  Bound by HBM: x read once, y written once.
#include "dsla_internal.cuh"

namespace dsla {

namespace {

constexpr int QN_THREADS = 256;

template <typename T> struct Eight;
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&x)[8]) {
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void zero() { a = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <int D, typename T, int NORM, bool INTERLEAVED>
__global__ void __launch_bounds__(QN_THREADS) qk_norm_rope_kernel(const dsla_qk_norm_rope_args p, int per) {
    constexpr int LANES = D / 8, HEADS = QN_THREADS / LANES;      // lanes per head, heads per CTA at a time
    constexpr int AHEAD = 4;                                      // rounds of heads whose loads are issued together
    __shared__ __align__(16) float scos[D / 2], ssin[D / 2];
    const int t = blockIdx.x, tid = threadIdx.x;
    const int lane = tid % LANES, first = 8 * lane;
    const int begin = blockIdx.y * per, end = min(begin + per, p.H + p.H_k);      // heads of this CTA, q's first
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int rot = p.rot, half = rot / 2;
    Eight<T> in[AHEAD];
    auto load = [&](int h0) {
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            const int h = h0 + r * HEADS + tid / LANES;
            if (h < end) in[r].load((h >= p.H ? reinterpret_cast<const T*>(p.k) + (size_t)t * p.k_stride + (size_t)(h - p.H) * D
                                              : reinterpret_cast<const T*>(p.q) + (size_t)t * p.q_stride + (size_t)h * D) + first);
            else in[r].zero();
        }
    };
    load(begin);
    // this lane's sines and cosines, with the sign that its half has: y = x cos + other sin
    float cs[8], sn[8];
    if (rot > 0) {
        if (tid < half) {
            const double turns = (double)p.positions[t] * (double)p.inv_freq[tid] * 0.31830988618379067154;      // half turns
            float a, b;
            sincospif((float)(turns - 2.0 * rint(0.5 * turns)), &a, &b);
            scos[tid] = b;
            ssin[tid] = a;
        }
        __syncthreads();
        if (first < rot) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int f = INTERLEAVED ? first / 2 + i / 2 : first >= half ? first - half + i : first + i;
                cs[i] = scos[f];
                sn[i] = (INTERLEAVED ? i % 2 == 0 : first < half) ? -ssin[f] : ssin[f];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
        }
    }
    const int step = half / 8;      // lanes between the halves
    const int partner = first < rot ? (first >= half ? (tid & 31) - step : (tid & 31) + step) : (tid & 31);
    for (int h0 = begin; h0 < end; h0 += AHEAD * HEADS) {
        if (h0 > begin) load(h0);
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            if (h0 + r * HEADS >= end) break;
            const int h = h0 + r * HEADS + tid / LANES;      // heads behind the last: zeros, not stored; the shuffles run in all lanes
            const bool is_k = h >= p.H;
            float x[8];
            in[r].get(x);
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
            const float* w = is_k ? p.k_weight : p.q_weight;
            if (w) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= __ldg(w + first + i);
            }
            if (rot > 0) {
                float other[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) other[i] = INTERLEAVED ? x[i ^ 1] : __shfl_sync(0xffffffffu, x[i], partner);
                if (first < rot) {      // channels that do not turn keep their bits
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], cs[i], other[i] * sn[i]);
                }
            }
            if (h < end) {
                T* dst = is_k ? reinterpret_cast<T*>(p.k_out) + (size_t)t * p.k_out_stride + (size_t)(h - p.H) * D
                              : reinterpret_cast<T*>(p.q_out) + (size_t)t * p.q_out_stride + (size_t)h * D;
                Eight<T>::store(dst + first, x);
            }
        }
    }
}

template <int D, typename T, int NORM>
cudaError_t launch_order(const cudaLaunchConfig_t* cfg, const dsla_qk_norm_rope_args& a, int per) {
    return a.interleaved ? cudaLaunchKernelEx(cfg, qk_norm_rope_kernel<D, T, NORM, true>, a, per)
                         : cudaLaunchKernelEx(cfg, qk_norm_rope_kernel<D, T, NORM, false>, a, per);
}
template <int D, typename T>
cudaError_t launch_norm(const cudaLaunchConfig_t* cfg, const dsla_qk_norm_rope_args& a, int per) {
    switch (a.norm) {
        case DSLA_NORM_RMS: return launch_order<D, T, DSLA_NORM_RMS>(cfg, a, per);
        case DSLA_NORM_L2: return launch_order<D, T, DSLA_NORM_L2>(cfg, a, per);
        default: return launch_order<D, T, DSLA_NORM_NONE>(cfg, a, per);
    }
}

}  // namespace

dsla_status launch_qk_norm_rope(const dsla_qk_norm_rope_args* a, cudaStream_t s) {
    const int total = a->H + a->H_k;
    const int at_once = QN_THREADS / (a->d / 8);
    const int per = total;
    const int parts = (total + per - 1) / per;
    (void)at_once;
    if (parts > 65535) return DSLA_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a->T, (unsigned)parts);
    cfg.blockDim = dim3(QN_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t rc;
    if (a->d == 128) rc = a->dtype == DSLA_BF16 ? launch_norm<128, __nv_bfloat16>(&cfg, *a, per) : launch_norm<128, float>(&cfg, *a, per);
    else rc = a->dtype == DSLA_BF16 ? launch_norm<64, __nv_bfloat16>(&cfg, *a, per) : launch_norm<64, float>(&cfg, *a, per);
    if (rc != cudaSuccess) return DSLA_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? DSLA_OK : DSLA_ERR_CUDA;
}

}  // namespace dsla
