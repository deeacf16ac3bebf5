// One token of the gated delta rule per batch row:
//     S <- g S,   u = beta (v - k S),   S <- S + k^T u,   o = scale q S .
// Each element of the fp32 state is read once and written once.  Both products with the state are taken from the loaded values, before the
// update: with y = k S_old and z = q S_old,
//     u = beta (v - g y),      o = scale (g z + (q.k) u),
// so one sum over d_k per column and product closes a step.  Bound by HBM: 8 d^2 bytes per (row, head).
#include "dsla_internal.cuh"

namespace dsla {

namespace {

// A CTA owns (row, head, 32 columns of d_v); a thread D / 16 rows of four columns, so that a warp's load covers four lines of
// 128 bytes; all loads of a CTA are in flight at once.  No atomics, one writer per element.
template <int D, typename T>
__global__ void __launch_bounds__(128) delta_decode_kernel(const DeltaParams p) {
    constexpr int SLABS = D / 32, RPT = D / 16;
    const int slab = blockIdx.x % SLABS;
    const int h = (blockIdx.x / SLABS) % p.H;
    const int b = blockIdx.x / (SLABS * p.H);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int c4 = tid & 7, r0 = tid >> 3;
    const int col = slab * 32 + c4 * 4;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (p.row_mask && p.row_mask[b] == 0) return;
    const int slot = p.slots ? p.slots[b] : b;
    const size_t base = ((size_t)b * p.H + h) * D;
    T* o = reinterpret_cast<T*>(p.o) + base;
    if (slot < 0 || slot >= p.num_slots) {
        if (tid < 32) o[slab * 32 + tid] = from_f32<T>(0.f);
        return;
    }
    float* S = p.state + ((size_t)slot * p.H + h) * (size_t)(D * D);
    float4 s[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) s[i] = __ldcs(reinterpret_cast<const float4*>(S + (size_t)(r0 + 16 * i) * D + col));

    __shared__ float sq[D], sk[D];
    __shared__ float red[4][2][32], redqk[4];
    const size_t qk_base = ((size_t)b * (p.H / p.group) + h / p.group) * D;
    float qk = 0.f;
    if (tid < D) {
        const float qv = to_f32(reinterpret_cast<const T*>(p.q)[qk_base + tid]) * p.scale, kv = to_f32(reinterpret_cast<const T*>(p.k)[qk_base + tid]);
        sq[tid] = qv;
        sk[tid] = kv;
        qk = qv * kv;
    }
    const float gate = p.gate[(size_t)b * p.H + h], g = gate < 0.f ? 0.f : gate, beta = p.beta[(size_t)b * p.H + h];
    const T* vp = reinterpret_cast<const T*>(p.v) + base + col;
    const float v0 = to_f32(vp[0]), v1 = to_f32(vp[1]), v2 = to_f32(vp[2]), v3 = to_f32(vp[3]);
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) qk += __shfl_xor_sync(0xffffffffu, qk, m);
    if (lane == 0) redqk[warp] = qk;
    __syncthreads();

    float y[4] = {0.f, 0.f, 0.f, 0.f}, z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const float kk = sk[r0 + 16 * i], qq = sq[r0 + 16 * i];
        y[0] = fmaf(kk, s[i].x, y[0]); y[1] = fmaf(kk, s[i].y, y[1]); y[2] = fmaf(kk, s[i].z, y[2]); y[3] = fmaf(kk, s[i].w, y[3]);
        z[0] = fmaf(qq, s[i].x, z[0]); z[1] = fmaf(qq, s[i].y, z[1]); z[2] = fmaf(qq, s[i].z, z[2]); z[3] = fmaf(qq, s[i].w, z[3]);
    }
    // over the 16 row groups: lanes that differ in bits 3 and 4, then the four warps
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int m = 8; m <= 16; m <<= 1) {
            y[j] += __shfl_xor_sync(0xffffffffu, y[j], m);
            z[j] += __shfl_xor_sync(0xffffffffu, z[j], m);
        }
    }
    if (lane < 8) {
        *reinterpret_cast<float4*>(&red[warp][0][lane * 4]) = make_float4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<float4*>(&red[warp][1][lane * 4]) = make_float4(z[0], z[1], z[2], z[3]);
    }
    __syncthreads();
    float u[4];
    const float vv[4] = {v0, v1, v2, v3};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = c4 * 4 + j;
        u[j] = beta * (vv[j] - g * (red[0][0][c] + red[1][0][c] + red[2][0][c] + red[3][0][c]));
    }
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const float kk = sk[r0 + 16 * i];
        float4 x = s[i];
        x.x = fmaf(g, x.x, kk * u[0]); x.y = fmaf(g, x.y, kk * u[1]); x.z = fmaf(g, x.z, kk * u[2]); x.w = fmaf(g, x.w, kk * u[3]);
        __stcs(reinterpret_cast<float4*>(S + (size_t)(r0 + 16 * i) * D + col), x);
    }
    if (tid < 8) {
        const float dot = redqk[0] + redqk[1] + redqk[2] + redqk[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c4 * 4 + j;
            const float zz = red[0][1][c] + red[1][1][c] + red[2][1][c] + red[3][1][c];
            o[slab * 32 + c] = from_f32<T>(fmaf(dot, u[j], g * zz));
        }
    }
}

template <int D, typename T>
cudaError_t launch(const cudaLaunchConfig_t* cfg, const DeltaParams& p) { return cudaLaunchKernelEx(cfg, delta_decode_kernel<D, T>, p); }

}  // namespace

dsla_status launch_delta_decode(const DeltaParams& p, int d, dsla_dtype dt, cudaStream_t s) {
    const long long blocks = (long long)p.N * p.H * (d / 32);
    if (blocks > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(128);
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
