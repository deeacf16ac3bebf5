// Gated delta rule over prompts in fp32, in chunks of 16 tokens (dsla_delta_tc.cu has the chunk's formulas):
//     R = V - G K S,       O = scale G Q S + (P T) R,       S <- G_15 S + Y R,       Y = K^T diag(D_15) T,   T = (I + A)^-1 diag(beta).
// A CTA owns (sequence, head, 16 columns of d_v).  Four warps walk the chunks; three groups of four make Y and P T of the chunks ahead in turn, and fetch their next one meanwhile.  The products with
// d_k or a chunk in their middle run as TF32 products of two terms (22 bits, fp32 sums): with plain FMAs each operand is read from shared memory as often as it is used, and the
// reads took 5600 cycles a chunk.  The state is fp32 in the accumulators' layout, one copy of it in shared memory for K S and Q S.  Products of gates are plain products: a gate of 0 is
// exact.  Tokens behind a sequence's end have no key, no beta and a gate of 1: they change nothing.
// Bound by the one SM that the walk and the preparation share: of the 35 us of 512 tokens of 4 heads of 64 the walk takes 23 by itself and the preparation 27 (issue slots 54 % busy; one group 68 us, two 54, four 35; operands stored as
// their two terms, so that nobody splits them twice, 46: the reads count; token by token, one shuffled sum per token and column, 63 to 112).  It serves fp32, and whoever asks for it; bf16 prompts have dsla_delta_tc.cu.
#include "dsla_delta.cuh"

namespace dsla {

namespace {

constexpr int DS_C = 16, DS_COLS = 16, DS_GROUPS = 3, DS_THREADS = 128 * (1 + DS_GROUPS), DS_BUFFERS = DS_GROUPS + 1;

// Four consecutive elements as fp32.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u));
}
// One chunk in shared memory; what the walk reads.  The pitches put the fragments' elements on different banks.
template <int D>
struct DeltaChunk {
    static constexpr int KP = D + 4, YP = D + 8, TP = DS_C + 4;
    float kq[2 * DS_C][KP];               // K, then Q
    float y[DS_C][YP];                    // Y transposed: [token][row of the state]
    float pt[DS_C][TP], v[DS_C][DS_COLS];
    float g[DS_C], sg[DS_C];              // G, scale G
};
// What the preparation keeps to itself.
struct DeltaWork {
    float a[DS_C][DS_C + 4], p[DS_C][DS_C + 4], t[DS_C][DS_C + 4], wt[DS_C][DS_C + 8], x[8][9];
    float power[4][DS_C];                 // products of 1, 2, 4, 8 gates, the last that of token j
    float beta[DS_C], left[DS_C];         // left: D_15,j
};
template <int D>
struct DeltaShared {
    static constexpr int SP = DS_COLS + 8;
    DeltaChunk<D> chunk[DS_BUFFERS];
    DeltaWork work[DS_GROUPS];
    float s[D][SP];                       // the state that the chunk starts from
    float r[DS_C][SP];                    // R
};

// Named barriers: 1 + group within the preparing groups, 4 within the walk; 5 + b: buffer b is ready (its group arrives, the walk waits), 9 + b: it has been walked.
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void pass_arrive(int id) { asm volatile("bar.arrive %0, 256;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void pass_wait(int id) { asm volatile("bar.sync %0, 256;" ::"r"(id) : "memory"); }

template <int D, typename T>
__global__ void __launch_bounds__(DS_THREADS) delta_simt_kernel(const DeltaParams p) {
    constexpr int SLABS = D / DS_COLS, TILES = D / 64;       // row tiles of the state of a warp: rows 16 (warp + 4 i) ..
    using Ch = DeltaChunk<D>;
    constexpr int LOADS = DS_C * D / 4 / 128;                // pieces of four channels of q, and of k, per preparing thread and chunk
    extern __shared__ __align__(16) uint8_t smem_raw[];
    DeltaShared<D>& sh = *reinterpret_cast<DeltaShared<D>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int slab = blockIdx.x % SLABS, h = (blockIdx.x / SLABS) % p.H, n = blockIdx.x / (SLABS * p.H);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t_begin = p.cu_seqlens ? p.cu_seqlens[n] : n * p.T, t_end = p.cu_seqlens ? p.cu_seqlens[n + 1] : t_begin + p.T;
    const int slot = p.slots ? p.slots[n] : n;
    if (slot < 0 || slot >= p.num_slots) return;
    const int len = t_end - t_begin;
    if (len <= 0 && p.use_initial_state) return;
    const int chunks = len > 0 ? (len + DS_C - 1) / DS_C : 0;

    if (warp >= 4) {
        // ---------------------------------------------------------------- preparation of every third chunk
        const int group = (warp - 4) >> 2, u = tid & 127, pw = warp & 3, Hqk = p.H / p.group, hq = h / p.group;
        const int i8 = 8 * (pw & 1), fr = lane >> 2, fq = lane & 3;
        DeltaWork& w = sh.work[group];
        float4 rq[LOADS], rk[LOADS], rv;
        float rg = 1.f, rb = 0.f;
        auto fetch = [&](int c) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int e = (i * 128 + u) * 4, t = c * DS_C + e / D;
                rq[i] = rk[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (t < len) {
                    const size_t at = ((size_t)(t_begin + t) * Hqk + hq) * D + e % D;
                    rq[i] = load4(reinterpret_cast<const T*>(p.q) + at);
                    rk[i] = load4(reinterpret_cast<const T*>(p.k) + at);
                }
            }
            if (u < DS_C * DS_COLS / 4) {
                const int t = c * DS_C + u / 4;
                rv = make_float4(0.f, 0.f, 0.f, 0.f);
                if (t < len) rv = load4(reinterpret_cast<const T*>(p.v) + ((size_t)(t_begin + t) * p.H + h) * D + slab * DS_COLS + (u & 3) * 4);
            } else if (u < 64 + DS_C) {
                const int t = c * DS_C + u - 64;
                rg = t < len ? p.gate[(size_t)(t_begin + t) * p.H + h] : 1.f;
                rb = t < len ? p.beta[(size_t)(t_begin + t) * p.H + h] : 0.f;
            }
        };
        fetch(group);
        for (int c = group; c < chunks; c += DS_GROUPS) {
            DeltaChunk<D>& ch = sh.chunk[c % DS_BUFFERS];
            {
                if (c >= DS_BUFFERS) pass_wait(9 + c % DS_BUFFERS);
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const int e = (i * 128 + u) * 4;
                    *reinterpret_cast<float4*>(&ch.kq[DS_C + e / D][e % D]) = rq[i];
                    *reinterpret_cast<float4*>(&ch.kq[e / D][e % D]) = rk[i];
                }
                if (u < 64) *reinterpret_cast<float4*>(&ch.v[u / 4][(u & 3) * 4]) = rv;
                else if (u < 96) {      // (one warp: lanes 0..15 have the gates)
                    const float one = rg < 0.f ? 0.f : rg;
                    const float two = one * __shfl_up_sync(0xffffffffu, one, 1), four = two * __shfl_up_sync(0xffffffffu, two, 2);
                    const float eight = four * __shfl_up_sync(0xffffffffu, four, 4);
                    float to = one, from = __shfl_down_sync(0xffffffffu, one, 1);
                    if (lane >= DS_C - 1) from = 1.f;
#pragma unroll
                    for (int off = 1; off < DS_C; off <<= 1) {
                        const float x = __shfl_up_sync(0xffffffffu, to, off), y = __shfl_down_sync(0xffffffffu, from, off);
                        if (lane >= off) to *= x;
                        if (lane + off < DS_C) from *= y;
                    }
                    if (lane < DS_C) {
                        w.power[0][lane] = one; w.power[1][lane] = two; w.power[2][lane] = four; w.power[3][lane] = eight;
                        w.beta[lane] = rb;
                        w.left[lane] = from;
                        ch.g[lane] = to;
                        ch.sg[lane] = to * p.scale;
                    }
                }
                fetch(c + DS_GROUPS);
                group_sync(1 + group);
                // warps 0, 1: k_j.k_i for 8 i each, 2, 3: q_j.k_i
                float f[4];
                product<D / 8>(f, ch.kq[pw < 2 ? 0 : DS_C], Ch::KP, 1, ch.kq[i8], 1, Ch::KP, 0, D / 8, lane);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int j = fr + 8 * half, i = i8 + 2 * fq, many = max(j - i - 1, 0);
                    float d1 = 1.f;      // D_j,i+1, from products of 1, 2, 4, 8 gates
                    int at = j;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float x = w.power[k][at];
                        const bool take = many >> k & 1;
                        d1 *= take ? x : 1.f;
                        at -= take ? 1 << k : 0;
                    }
                    const float next = w.power[0][i + 1];
                    const float d0 = i < j ? d1 * next : 1.f, x0 = f[2 * half], x1 = f[2 * half + 1];
                    if (pw < 2) {
                        const float beta = w.beta[j];
                        w.a[j][i] = i < j ? beta * d0 * x0 : 0.f;
                        w.a[j][i + 1] = i + 1 < j ? beta * d1 * x1 : 0.f;
                    } else {
                        w.p[j][i] = i <= j ? p.scale * d0 * x0 : 0.f;
                        w.p[j][i + 1] = i < j ? p.scale * d1 * x1 : 0.f;
                    }
                }
                group_sync(1 + group);
                // (I + A)^-1: two blocks of 8 by substitution (thread = column), then -c^-1 b a^-1 below them
                if (u < 16) {
                    const int b = u & 8, col = u & 7;
                    float4 a[8][2];
#pragma unroll
                    for (int i = 1; i < 8; ++i) {
                        a[i][0] = *reinterpret_cast<const float4*>(&w.a[b + i][b]);
                        a[i][1] = *reinterpret_cast<const float4*>(&w.a[b + i][b + 4]);
                    }
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float s0 = i == col ? 1.f : 0.f, s1 = 0.f;
                        if (i > 0) s0 = fmaf(-a[i][0].x, x[0], s0);
                        if (i > 1) s1 = fmaf(-a[i][0].y, x[1], s1);
                        if (i > 2) s0 = fmaf(-a[i][0].z, x[2], s0);
                        if (i > 3) s1 = fmaf(-a[i][0].w, x[3], s1);
                        if (i > 4) s0 = fmaf(-a[i][1].x, x[4], s0);
                        if (i > 5) s1 = fmaf(-a[i][1].y, x[5], s1);
                        if (i > 6) s0 = fmaf(-a[i][1].z, x[6], s0);
                        x[i] = s0 + s1;
                        w.t[b + i][b + col] = x[i];
                        if (b == 0) w.t[i][8 + col] = 0.f;
                    }
                }
                group_sync(1 + group);
                if (u < 64) {
                    const int i = u >> 3, k = u & 7;
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = fmaf(w.a[8 + i][e], w.t[e][k], s);
                    w.x[i][k] = s;
                }
                group_sync(1 + group);
                if (u < 64) {
                    const int i = u >> 3, k = u & 7;
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = fmaf(-w.t[8 + i][8 + e], w.x[e][k], s);
                    w.t[8 + i][k] = s;
                }
                group_sync(1 + group);
#pragma unroll
                for (int r = 0; r < 2; ++r) {      // T = inverse diag(beta), and its rows weighted
                    const int s = u >> 3, t = 2 * (u & 7) + r;
                    const float x = w.t[s][t] * w.beta[t];
                    w.t[s][t] = x;
                    w.wt[s][t] = x * w.left[s];
                }
                group_sync(1 + group);
                // Y transposed = (diag(D_15) T)^T K: D / 4 of its columns a warp; P T: 8 columns each of warps 0, 1
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const int n0 = 8 * (pw * (D / 32) + i);
                    product<2>(f, &w.wt[0][0], 1, DS_C + 8, &ch.kq[0][n0], Ch::KP, 1, 0, 2, lane);
                    put_fragment(&ch.y[0][n0], Ch::YP, f, 1.f, lane);
                }
                if (pw < 2) {
                    product<2>(f, &w.p[0][0], DS_C + 4, 1, &w.t[0][i8], DS_C + 4, 1, i8 / 8, 2, lane);
                    put_fragment(&ch.pt[0][i8], Ch::TP, f, 1.f, lane);
                }
            }
            pass_arrive(5 + c % DS_BUFFERS);
        }
        return;
    }

    // -------------------------------------------------------------------- the walk
    const int fr = lane >> 2, fq = lane & 3;
    float* S = p.state + ((size_t)slot * p.H + h) * (size_t)(D * D) + slab * DS_COLS;
    float s[TILES][2][4];      // rows 16 (warp + 4 i) + fr (+ 8), columns 8 k + 2 fq (+ 1)
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float2 x = make_float2(0.f, 0.f);
                if (p.use_initial_state) x = *reinterpret_cast<const float2*>(S + (size_t)(16 * (warp + 4 * i) + fr + 8 * e) * D + 8 * k + 2 * fq);
                s[i][k][2 * e] = x.x;
                s[i][k][2 * e + 1] = x.y;
            }
    T* o = reinterpret_cast<T*>(p.o) + ((size_t)t_begin * p.H + h) * D + slab * DS_COLS;
    const int n0 = 8 * (warp & 1);      // this warp's columns of K S (warps 0, 1) or Q S (2, 3)
    for (int c = 0; c < chunks; ++c) {
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) put_fragment(&sh.s[16 * (warp + 4 * i)][8 * k], DeltaShared<D>::SP, s[i][k], 1.f, lane);
        pass_wait(5 + c % DS_BUFFERS);      // chunk c is ready, and so is S
        const Ch& ch = sh.chunk[c % DS_BUFFERS];
        float f[4];
        product<D / 8>(f, ch.kq[warp < 2 ? 0 : DS_C], Ch::KP, 1, &sh.s[0][n0], DeltaShared<D>::SP, 1, 0, D / 8, lane);
        if (warp < 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = fr + 8 * (e >> 1), col = n0 + 2 * fq + (e & 1);
                f[e] = fmaf(-ch.g[t], f[e], ch.v[t][col]);
            }
            put_fragment(&sh.r[0][n0], DeltaShared<D>::SP, f, 1.f, lane);
        }
        group_sync(4);
        const float last = ch.g[DS_C - 1];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float d[4];
                product<2>(d, &ch.y[0][16 * (warp + 4 * i)], 1, Ch::YP, &sh.r[0][8 * k], DeltaShared<D>::SP, 1, 0, 2, lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][k][e] = fmaf(last, s[i][k][e], d[e]);
            }
        if (warp >= 2) {
            float d[4];
            product<2>(d, &ch.pt[0][0], Ch::TP, 1, &sh.r[0][n0], DeltaShared<D>::SP, 1, 0, 2, lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = fr + 8 * (e >> 1), col = n0 + 2 * fq + (e & 1);
                if (c * DS_C + t < len) o[(size_t)(c * DS_C + t) * p.H * D + col] = from_f32<T>(fmaf(ch.sg[t], f[e], d[e]));
            }
        }
        if (c + DS_BUFFERS < chunks) pass_arrive(9 + c % DS_BUFFERS);
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<float2*>(S + (size_t)(16 * (warp + 4 * i) + fr + 8 * e) * D + 8 * k + 2 * fq) = make_float2(s[i][k][2 * e], s[i][k][2 * e + 1]);
}

template <int D, typename T>
cudaError_t launch(cudaLaunchConfig_t* cfg, const DeltaParams& p) {
    const cudaError_t rc = cudaFuncSetAttribute(delta_simt_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(DeltaShared<D>));
    if (rc != cudaSuccess) return rc;
    cfg->dynamicSmemBytes = sizeof(DeltaShared<D>);
    return cudaLaunchKernelEx(cfg, delta_simt_kernel<D, T>, p);
}

}  // namespace

dsla_status launch_delta_simt(const DeltaParams& p, int d, dsla_dtype dt, cudaStream_t s) {
    const long long blocks = (long long)p.N * p.H * (d / DS_COLS);
    if (blocks > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(DS_THREADS);
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
