// Gated delta rule over prompts, token by token on CUDA cores in fp32.  With S' the state before token t - 1,
//     y = k_t S = g_{t-1} (k_t S') + (k_t.k_{t-1}) u_{t-1},     z = q_t S = g_{t-1} (q_t S') + (q_t.k_{t-1}) u_{t-1},
//     u_t = beta_t (v_t - g_t y),     o_t = scale (g_t z + (q_t.k_t) u_t),     S <- g_t S + k_t^T u_t :
// the sums over d_k that token t needs are taken from the state one token earlier, so they run while token t - 1 is still being finished, and only
// two products lie between one u and the next.  (Sums from the state itself, four threads to a column: 112 us for 512 tokens of 4 heads of 64.)
// A CTA owns (sequence, head, 16 columns of d_v); eight threads share a column, each with D / 8 rows of it in registers.  Tokens are staged in blocks as fp32,
// three blocks deep in shared memory, and one more on its way in registers; behind a sequence's end they are tokens without keys, which change
// nothing.  Bound by that chain: it serves fp32 (whose products the tensor cores do not take) and whoever asks for it; bf16 prompts have the
// chunks of dsla_delta_tc.cu.
#include "dsla_internal.cuh"

namespace dsla {

namespace {

constexpr int DR_THREADS = 128, DR_COLS = 16, DR_PARTS = 8;

// Four consecutive elements as fp32.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u));
}
// Pairs of fp32: one instruction for two.
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ float sum2(uint64_t x, uint64_t y) {
    float a, b, c, d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(c), "=f"(d) : "l"(y));
    return (a + b) + (c + d);
}
__device__ __forceinline__ float over_parts(float x) {      // lanes 4 part + column
    x += __shfl_xor_sync(0xffffffffu, x, 4);
    x += __shfl_xor_sync(0xffffffffu, x, 8);
    return x + __shfl_xor_sync(0xffffffffu, x, 16);
}

template <int D, typename T>
__global__ void __launch_bounds__(DR_THREADS) delta_recurrent_kernel(const DeltaParams p) {
    constexpr int BLOCK = 1024 / D;                        // tokens staged at a time
    constexpr int SLABS = D / DR_COLS, PIECES = D / (4 * DR_PARTS);      // a thread's rows: 32 i + 4 part .. + 3
    constexpr int LOADS = BLOCK * D / 4 / DR_THREADS;      // 16-byte pieces of q, and of k, per thread and block
    __shared__ __align__(16) float sq[3][BLOCK][D], sk[3][BLOCK][D];
    __shared__ float sv[3][BLOCK][DR_COLS], sg[3][BLOCK], sb[3][BLOCK];
    __shared__ float skk[3][BLOCK], sqk1[3][BLOCK], sqk[3][BLOCK];      // k_t.k_{t-1}, q_t.k_{t-1}, q_t.k_t
    const int tid = threadIdx.x, lane = tid & 31;
    const int slab = blockIdx.x % SLABS;
    const int h = (blockIdx.x / SLABS) % p.H;
    const int n = blockIdx.x / (SLABS * p.H);
    const int part = lane >> 2, c = (tid >> 5) * 4 + (lane & 3), col = slab * DR_COLS + c;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t_begin = p.cu_seqlens ? p.cu_seqlens[n] : n * p.T, t_end = p.cu_seqlens ? p.cu_seqlens[n + 1] : t_begin + p.T;
    const int slot = p.slots ? p.slots[n] : n;
    if (slot < 0 || slot >= p.num_slots) return;
    const int len = t_end - t_begin;
    if (len <= 0 && p.use_initial_state) return;
    const int Hqk = p.H / p.group, hq = h / p.group;
    float* S = p.state + ((size_t)slot * p.H + h) * (size_t)(D * D) + col;
    uint64_t s[2 * PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (p.use_initial_state) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = S[(size_t)(32 * i + 4 * part + e) * D];
        }
        s[2 * i] = pair(x[0], x[1]);
        s[2 * i + 1] = pair(x[2], x[3]);
    }

    float4 rq[LOADS], rk[LOADS], rv;
    float rg = 1.f, rb = 0.f;
    auto fetch = [&](int blk) {      // block blk of the sequence into registers
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int e = (i * DR_THREADS + tid) * 4, t = blk * BLOCK + e / D;
            rq[i] = rk[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (t < len) {
                const size_t at = ((size_t)(t_begin + t) * Hqk + hq) * D + e % D;
                rq[i] = load4(reinterpret_cast<const T*>(p.q) + at);
                rk[i] = load4(reinterpret_cast<const T*>(p.k) + at);
            }
        }
        if (tid < BLOCK * DR_COLS / 4) {
            const int t = blk * BLOCK + tid / 4;
            rv = make_float4(0.f, 0.f, 0.f, 0.f);
            if (t < len) rv = load4(reinterpret_cast<const T*>(p.v) + ((size_t)(t_begin + t) * p.H + h) * D + slab * DR_COLS + (tid & 3) * 4);
        }
        if (tid < BLOCK) {
            const int t = blk * BLOCK + tid;
            rg = t < len ? p.gate[(size_t)(t_begin + t) * p.H + h] : 1.f;
            rb = t < len ? p.beta[(size_t)(t_begin + t) * p.H + h] : 0.f;
        }
    };
    auto put = [&](int blk) {
        const int buf = blk % 3;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int e = (i * DR_THREADS + tid) * 4;
            rq[i].x *= p.scale; rq[i].y *= p.scale; rq[i].z *= p.scale; rq[i].w *= p.scale;
            *reinterpret_cast<float4*>(&sq[buf][e / D][e % D]) = rq[i];
            *reinterpret_cast<float4*>(&sk[buf][e / D][e % D]) = rk[i];
        }
        if (tid < BLOCK * DR_COLS / 4) *reinterpret_cast<float4*>(&sv[buf][tid / 4][(tid & 3) * 4]) = rv;
        if (tid < BLOCK) {
            sg[buf][tid] = rg < 0.f ? 0.f : rg;
            sb[buf][tid] = rb;
        }
    };
    auto dots = [&](int blk) {       // products of a block's keys and queries with each other; 128 / BLOCK threads to a token
        constexpr int PER = DR_THREADS / BLOCK;
        const int buf = blk % 3, t = tid / PER;
        const float* before = t > 0 ? sk[buf][t - 1] : sk[(blk + 2) % 3][BLOCK - 1];
        float a = 0.f, b = 0.f, d = 0.f;
#pragma unroll
        for (int i = 0; i < D / (4 * PER); ++i) {
            const int at = 4 * (i * PER + tid % PER);
            const float4 k = *reinterpret_cast<const float4*>(&sk[buf][t][at]), q = *reinterpret_cast<const float4*>(&sq[buf][t][at]);
            const float4 o = *reinterpret_cast<const float4*>(before + at);
            a += k.x * o.x + k.y * o.y + k.z * o.z + k.w * o.w;
            b += q.x * o.x + q.y * o.y + q.z * o.z + q.w * o.w;
            d += q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
        }
#pragma unroll
        for (int m = 1; m < PER; m <<= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, m);
            b += __shfl_xor_sync(0xffffffffu, b, m);
            d += __shfl_xor_sync(0xffffffffu, d, m);
        }
        if (tid % PER == 0) {
            const bool first = blk == 0 && t == 0;      // no token before it
            skk[buf][t] = first ? 0.f : a;
            sqk1[buf][t] = first ? 0.f : b;
            sqk[buf][t] = d;
        }
    };
    const int blocks = (len + BLOCK - 1) / BLOCK;
    float u = 0.f, g = 1.f, ya = 0.f, za = 0.f;      // of the token before: u, gate; of this one: k and q times the state before that token
    const float* kp = sk[2][BLOCK - 1];               // the key of the token before
    auto sums = [&](const float* k, const float* q) {
        uint64_t y0 = 0, y1 = 0, z0 = 0, z1 = 0;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const ulonglong2 kk = *reinterpret_cast<const ulonglong2*>(k + 32 * i + 4 * part), qq = *reinterpret_cast<const ulonglong2*>(q + 32 * i + 4 * part);
            y0 = fma2(kk.x, s[2 * i], y0); y1 = fma2(kk.y, s[2 * i + 1], y1);
            z0 = fma2(qq.x, s[2 * i], z0); z1 = fma2(qq.y, s[2 * i + 1], z1);
        }
        ya = over_parts(sum2(y0, y1));
        za = over_parts(sum2(z0, z1));
    };
    auto advance = [&]() {           // the state takes in the token before
        const uint64_t gg = pair(g, g), uu = pair(u, u);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const ulonglong2 kk = *reinterpret_cast<const ulonglong2*>(kp + 32 * i + 4 * part);
            s[2 * i] = fma2(kk.x, uu, mul2(gg, s[2 * i]));
            s[2 * i + 1] = fma2(kk.y, uu, mul2(gg, s[2 * i + 1]));
        }
    };
    if (blocks > 0) {
        fetch(0);
        put(0);
        fetch(1);
        put(1);
        if (tid < D) sk[2][BLOCK - 1][tid] = 0.f;
        __syncthreads();
        dots(0);
        dots(1);
        fetch(2);
        sums(sk[0][0], sq[0][0]);
        __syncthreads();
    }
    T* o = reinterpret_cast<T*>(p.o) + ((size_t)t_begin * p.H + h) * D + col;
    const size_t step = (size_t)p.H * D;
    for (int blk = 0; blk < blocks; ++blk) {
        const int buf = blk % 3, next = (blk + 1) % 3, left = len - blk * BLOCK;
#pragma unroll
        for (int t = 0; t < BLOCK; ++t) {
            const float gt = sg[buf][t], bt = sb[buf][t];
            const float y = fmaf(skk[buf][t], u, g * ya), z = fmaf(sqk1[buf][t], u, g * za);
            advance();
            kp = sk[buf][t];
            if (t + 1 < BLOCK) sums(sk[buf][t + 1], sq[buf][t + 1]);
            else sums(sk[next][0], sq[next][0]);
            u = bt * fmaf(-gt, y, sv[buf][t][c]);
            g = gt;
            if (part == 0 && t < left) o[(size_t)t * step] = from_f32<T>(fmaf(sqk[buf][t], u, gt * z));
        }
        o += (size_t)BLOCK * step;
        __syncthreads();
        if (blk + 2 < blocks + 1) {      // (the last block still looks one token ahead)
            put(blk + 2);
            fetch(blk + 3);
            __syncthreads();
            dots(blk + 2);
            __syncthreads();
        }
    }
    if (blocks > 0) advance();
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x, y;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(s[2 * i + e]));
            S[(size_t)(32 * i + 4 * part + 2 * e) * D] = x;
            S[(size_t)(32 * i + 4 * part + 2 * e + 1) * D] = y;
        }
    }
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
