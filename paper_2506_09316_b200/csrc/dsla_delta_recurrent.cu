// Gated delta rule over prompts, token by token on CUDA cores in fp32.  With S" the state before token t - 2,
//     k_t S = g_{t-1} (g_{t-2} (k_t S") + (k_t.k_{t-2}) u_{t-2}) + (k_t.k_{t-1}) u_{t-1}     and the same with q_t,
//     u_t = beta_t (v_t - g_t k_t S),     o_t = scale (g_t q_t S + (q_t.k_t) u_t),     S <- g_t S + k_t^T u_t :
// the sums over d_k that token t needs are taken from the state two tokens earlier, so their reduction runs while the tokens before t are being finished, and
// only two products lie between one u and the next.  (512 tokens of 4 heads of 64: sums from the state itself 112 us, from one token earlier 65 us.)
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
    __shared__ float4 sc[3][BLOCK];                                         // k_t.k_{t-1}, k_t.k_{t-2}, q_t.k_{t-1}, q_t.k_{t-2}
    __shared__ float sqk[3][BLOCK];                                         // q_t.k_t
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
        const int buf = blk % 3, t = tid / PER, before = (blk + 2) % 3;
        const float* one = t > 0 ? sk[buf][t - 1] : sk[before][BLOCK - 1];
        const float* two = t > 1 ? sk[buf][t - 2] : sk[before][BLOCK - 2 + t];
        float x[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / (4 * PER); ++i) {
            const int at = 4 * (i * PER + tid % PER);
            const float4 k = *reinterpret_cast<const float4*>(&sk[buf][t][at]), q = *reinterpret_cast<const float4*>(&sq[buf][t][at]);
            const float4 a = *reinterpret_cast<const float4*>(one + at), b = *reinterpret_cast<const float4*>(two + at);
            x[0] += k.x * a.x + k.y * a.y + k.z * a.z + k.w * a.w;
            x[1] += k.x * b.x + k.y * b.y + k.z * b.z + k.w * b.w;
            x[2] += q.x * a.x + q.y * a.y + q.z * a.z + q.w * a.w;
            x[3] += q.x * b.x + q.y * b.y + q.z * b.z + q.w * b.w;
            x[4] += q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
        }
#pragma unroll
        for (int m = 1; m < PER; m <<= 1)
#pragma unroll
            for (int i = 0; i < 5; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], m);
        if (tid % PER == 0) {
            sc[buf][t] = make_float4(x[0], x[1], x[2], x[3]);
            sqk[buf][t] = x[4];
        }
    };
    const int blocks = (len + BLOCK - 1) / BLOCK;
    float u1 = 0.f, g1 = 1.f, u2 = 0.f, g2 = 1.f;      // of the two tokens before this one
    float ya = 0.f, za = 0.f, py = 0.f, pz = 0.f;      // this token's sums; this thread's part of the next one's
    const float* kp = sk[2][BLOCK - 1];                 // the key of the token before
    auto sums = [&](const float* k, const float* q) {
        uint64_t y0 = 0, y1 = 0, z0 = 0, z1 = 0;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const ulonglong2 kk = *reinterpret_cast<const ulonglong2*>(k + 32 * i + 4 * part), qq = *reinterpret_cast<const ulonglong2*>(q + 32 * i + 4 * part);
            y0 = fma2(kk.x, s[2 * i], y0); y1 = fma2(kk.y, s[2 * i + 1], y1);
            z0 = fma2(qq.x, s[2 * i], z0); z1 = fma2(qq.y, s[2 * i + 1], z1);
        }
        py = sum2(y0, y1);
        pz = sum2(z0, z1);
    };
    auto advance = [&]() {           // the state takes in the token before
        const uint64_t gg = pair(g1, g1), uu = pair(u1, u1);
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
        for (int i = tid; i < 2 * D; i += DR_THREADS) sk[2][BLOCK - 2 + i / D][i % D] = 0.f;      // no tokens before the first
        __syncthreads();
        dots(0);
        dots(1);
        fetch(2);
        sums(sk[0][0], sq[0][0]);
        ya = over_parts(py);
        za = over_parts(pz);
        sums(sk[0][1], sq[0][1]);
        __syncthreads();
    }
    T* o = reinterpret_cast<T*>(p.o) + ((size_t)t_begin * p.H + h) * D + col;
    const size_t step = (size_t)p.H * D;
    for (int blk = 0; blk < blocks; ++blk) {
        const int buf = blk % 3, next = (blk + 1) % 3, left = len - blk * BLOCK;
#pragma unroll
        for (int t = 0; t < BLOCK; ++t) {
            const float4 c4 = sc[buf][t];
            const float gt = sg[buf][t], bt = sb[buf][t];
            const float yb = g1 * fmaf(c4.y, u2, g2 * ya), zb = g1 * fmaf(c4.w, u2, g2 * za);
            // the next token's sums close, the state takes in the token before, the sums of the token after next begin
            float cy = py, cz = pz;
            cy += __shfl_xor_sync(0xffffffffu, cy, 4);
            cz += __shfl_xor_sync(0xffffffffu, cz, 4);
            advance();
            cy += __shfl_xor_sync(0xffffffffu, cy, 8);
            cz += __shfl_xor_sync(0xffffffffu, cz, 8);
            if (t + 2 < BLOCK) sums(sk[buf][t + 2], sq[buf][t + 2]);
            else sums(sk[next][t + 2 - BLOCK], sq[next][t + 2 - BLOCK]);
            cy += __shfl_xor_sync(0xffffffffu, cy, 16);
            cz += __shfl_xor_sync(0xffffffffu, cz, 16);
            const float u = bt * fmaf(-gt, fmaf(c4.x, u1, yb), sv[buf][t][c]), z = fmaf(c4.z, u1, zb);
            if (part == 0 && t < left) o[(size_t)t * step] = from_f32<T>(fmaf(sqk[buf][t], u, gt * z));
            ya = cy;
            za = cz;
            u2 = u1; g2 = g1;
            u1 = u; g1 = gt;
            kp = sk[buf][t];
        }
        o += (size_t)BLOCK * step;
        __syncthreads();
        if (blk + 1 < blocks) {      // (the last block still looks two tokens ahead)
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
