// Gated delta rule over prompts, token by token on CUDA cores in fp32 (dsla_delta_decode.cu has the step's two sums):
//     y = k S,  z = q S,   u = beta (v - g y),   o = scale (g z + (q.k) u),   S <- g S + k^T u .
// A CTA owns (sequence, head, 32 columns of d_v); four threads share a column, each with D / 4 rows of it in registers, so a token's
// chain is a short dot product, two shuffles and the update.  Tokens are staged 16 at a time in shared memory as fp32, two buffers, the next
// block on its way into registers while one is worked on.  Bound by that chain: it serves fp32 (whose products the tensor cores do not
// take) and whoever asks for it; bf16 prompts have the chunks of dsla_delta_tc.cu.
#include "dsla_internal.cuh"

namespace dsla {

namespace {

constexpr int DR_THREADS = 128, DR_BLOCK = 16, DR_COLS = 32;

// Four consecutive elements as fp32.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u));
}

template <int D, typename T>
__global__ void __launch_bounds__(DR_THREADS) delta_recurrent_kernel(const DeltaParams p) {
    constexpr int SLABS = D / DR_COLS, ROWS = D / 4, PIECES = ROWS / 4;      // a thread's rows: 16 i + 4 part .. + 3
    constexpr int QK_LOADS = DR_BLOCK * D / 4 / DR_THREADS;                  // 16-byte (fp32) pieces of q, and of k, per thread and block
    __shared__ __align__(16) float sq[2][DR_BLOCK][D], sk[2][DR_BLOCK][D], sv[2][DR_BLOCK][DR_COLS];
    __shared__ float sg[2][DR_BLOCK], sb[2][DR_BLOCK], sdot[2][DR_BLOCK];
    const int tid = threadIdx.x;
    const int slab = blockIdx.x % SLABS;
    const int h = (blockIdx.x / SLABS) % p.H;
    const int n = blockIdx.x / (SLABS * p.H);
    const int part = tid & 3, c = tid >> 2, col = slab * DR_COLS + c;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t_begin = p.cu_seqlens ? p.cu_seqlens[n] : n * p.T, t_end = p.cu_seqlens ? p.cu_seqlens[n + 1] : t_begin + p.T;
    const int slot = p.slots ? p.slots[n] : n;
    if (slot < 0 || slot >= p.num_slots) return;
    const int len = t_end - t_begin;
    if (len <= 0 && p.use_initial_state) return;
    const int Hqk = p.H / p.group, hq = h / p.group;
    float* S = p.state + ((size_t)slot * p.H + h) * (size_t)(D * D) + col;
    float s[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) s[i] = p.use_initial_state ? S[(size_t)(16 * (i >> 2) + 4 * part + (i & 3)) * D] : 0.f;

    float4 rq[QK_LOADS], rk[QK_LOADS], rv;
    float rg = 1.f, rb = 0.f;
    // Block blk of the sequence into registers; tokens behind the end stay zero and are not worked on.
    auto fetch = [&](int blk) {
#pragma unroll
        for (int i = 0; i < QK_LOADS; ++i) {
            const int e = (i * DR_THREADS + tid) * 4, t = blk * DR_BLOCK + e / D;
            rq[i] = rk[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (t < len) {
                const size_t at = ((size_t)(t_begin + t) * Hqk + hq) * D + e % D;
                rq[i] = load4(reinterpret_cast<const T*>(p.q) + at);
                rk[i] = load4(reinterpret_cast<const T*>(p.k) + at);
            }
        }
        {
            const int t = blk * DR_BLOCK + tid / 8;
            rv = make_float4(0.f, 0.f, 0.f, 0.f);
            if (t < len) rv = load4(reinterpret_cast<const T*>(p.v) + ((size_t)(t_begin + t) * p.H + h) * D + slab * DR_COLS + (tid & 7) * 4);
        }
        const int t = blk * DR_BLOCK + (tid & (DR_BLOCK - 1));
        if (tid < DR_BLOCK) rg = t < len ? p.gate[(size_t)(t_begin + t) * p.H + h] : 1.f;
        else if (tid < 2 * DR_BLOCK) rb = t < len ? p.beta[(size_t)(t_begin + t) * p.H + h] : 0.f;
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < QK_LOADS; ++i) {
            const int e = (i * DR_THREADS + tid) * 4;
            rq[i].x *= p.scale; rq[i].y *= p.scale; rq[i].z *= p.scale; rq[i].w *= p.scale;
            *reinterpret_cast<float4*>(&sq[buf][e / D][e % D]) = rq[i];
            *reinterpret_cast<float4*>(&sk[buf][e / D][e % D]) = rk[i];
            float dot = rq[i].x * rk[i].x + rq[i].y * rk[i].y + rq[i].z * rk[i].z + rq[i].w * rk[i].w;      // D / 4 neighbouring threads hold a token
#pragma unroll
            for (int m = 1; m < D / 4; m <<= 1) dot += __shfl_xor_sync(0xffffffffu, dot, m);
            if (tid % (D / 4) == 0) sdot[buf][e / D] = dot;
        }
        *reinterpret_cast<float4*>(&sv[buf][tid / 8][(tid & 7) * 4]) = rv;
        if (tid < DR_BLOCK) sg[buf][tid] = rg < 0.f ? 0.f : rg;
        else if (tid < 2 * DR_BLOCK) sb[buf][tid - DR_BLOCK] = rb;
    };
    const int blocks = (len + DR_BLOCK - 1) / DR_BLOCK;
    if (blocks > 0) {
        fetch(0);
        put(0);
    }
    __syncthreads();
    T* o = reinterpret_cast<T*>(p.o) + ((size_t)t_begin * p.H + h) * D + col;
    for (int blk = 0; blk < blocks; ++blk) {
        const int buf = blk & 1, count = min(DR_BLOCK, len - blk * DR_BLOCK);
        if (blk + 1 < blocks) fetch(blk + 1);
        for (int t = 0; t < count; ++t) {
            float y[4] = {0.f, 0.f, 0.f, 0.f}, z[4] = {0.f, 0.f, 0.f, 0.f};
            float4 kk[PIECES];
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                kk[i] = *reinterpret_cast<const float4*>(&sk[buf][t][16 * i + 4 * part]);
                const float4 qq = *reinterpret_cast<const float4*>(&sq[buf][t][16 * i + 4 * part]);
                y[0] = fmaf(kk[i].x, s[4 * i], y[0]); y[1] = fmaf(kk[i].y, s[4 * i + 1], y[1]);
                y[2] = fmaf(kk[i].z, s[4 * i + 2], y[2]); y[3] = fmaf(kk[i].w, s[4 * i + 3], y[3]);
                z[0] = fmaf(qq.x, s[4 * i], z[0]); z[1] = fmaf(qq.y, s[4 * i + 1], z[1]);
                z[2] = fmaf(qq.z, s[4 * i + 2], z[2]); z[3] = fmaf(qq.w, s[4 * i + 3], z[3]);
            }
            float ys = (y[0] + y[1]) + (y[2] + y[3]), zs = (z[0] + z[1]) + (z[2] + z[3]);
            ys += __shfl_xor_sync(0xffffffffu, ys, 1);
            zs += __shfl_xor_sync(0xffffffffu, zs, 1);
            ys += __shfl_xor_sync(0xffffffffu, ys, 2);
            zs += __shfl_xor_sync(0xffffffffu, zs, 2);
            const float g = sg[buf][t];
            const float u = sb[buf][t] * (sv[buf][t][c] - g * ys);
            if (part == 0) o[(size_t)(blk * DR_BLOCK + t) * p.H * D] = from_f32<T>(fmaf(sdot[buf][t], u, g * zs));
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                s[4 * i] = fmaf(g, s[4 * i], kk[i].x * u); s[4 * i + 1] = fmaf(g, s[4 * i + 1], kk[i].y * u);
                s[4 * i + 2] = fmaf(g, s[4 * i + 2], kk[i].z * u); s[4 * i + 3] = fmaf(g, s[4 * i + 3], kk[i].w * u);
            }
        }
        if (blk + 1 < blocks) put(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) S[(size_t)(16 * (i >> 2) + 4 * part + (i & 3)) * D] = s[i];
}

template <int D, typename T>
cudaError_t launch(const cudaLaunchConfig_t* cfg, const DeltaParams& p) { return cudaLaunchKernelEx(cfg, delta_recurrent_kernel<D, T>, p); }

}  // namespace

dsla_status launch_delta_recurrent(const DeltaParams& p, int d, dsla_dtype dt, cudaStream_t s) {
    const long long blocks = (long long)p.N * p.H * (d / DR_COLS);
    if (blocks > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(DR_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t rc;
    if (d == 128) rc = dt == DSLA_BF16 ? launch<128, __nv_bfloat16>(&cfg, p) : launch<128, float>(&cfg, p);
    else rc = dt == DSLA_BF16 ? launch<64, __nv_bfloat16>(&cfg, p) : launch<64, float>(&cfg, p);
    if (rc != cudaSuccess) return DSLA_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? DSLA_OK : DSLA_ERR_CUDA;
}

}  // namespace dsla
