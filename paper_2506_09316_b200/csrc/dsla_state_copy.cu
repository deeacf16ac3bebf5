// Copying, forking, compacting and freeing slots of a state store: a list of moves (source slot, target slot) with the result of
// carrying them out one after the other.  Every thread owns places (16 bytes) of a slot and walks the whole list for each,
// so the order of the moves is the order of one thread's loads and stores and needs no synchronisation across the grid, whatever slots
// the list names.  Moves are taken eight at a time; the loads of eight are all issued before the first store unless one of them
// reads what an earlier of the eight writes.  Bound by HBM: sources read once, targets written once.
#include "dsla_internal.cuh"

namespace dsla {

namespace {

constexpr int SC_THREADS = 128, SC_LIST = 256, SC_GROUP = 8;
enum : int { SC_SKIP = -2, SC_CLEAR = -1 };

__global__ void __launch_bounds__(SC_THREADS) state_copy_kernel(float4* data, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int n,
                                                                int num_slots, size_t slot4) {
    __shared__ int from[SC_LIST], to[SC_LIST];
    __shared__ uint8_t chained[SC_LIST / SC_GROUP];      // some move of the group reads the target of an earlier one of it
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const size_t at = (size_t)blockIdx.x * SC_THREADS + threadIdx.x;
    float4* const place = data + at;
    for (int first = 0; first < n; first += SC_LIST) {
        const int count = min(SC_LIST, n - first);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < SC_LIST / SC_THREADS; ++r) {
            const int i = r * SC_THREADS + threadIdx.x;
            int a = i < count ? src[first + i] : SC_SKIP;
            const int b = i < count ? dst[first + i] : 0;
            if (a < -1 || a >= num_slots || b < 0 || b >= num_slots || a == b) a = SC_SKIP;
            from[i] = a;
            to[i] = b;
            bool c = false;      // the lanes of a group compare with those before them
#pragma unroll
            for (int k = 1; k < SC_GROUP; ++k) {
                const int fa = __shfl_up_sync(0xffffffffu, a, k), tb = __shfl_up_sync(0xffffffffu, b, k);
                c |= (int)(threadIdx.x % SC_GROUP) >= k && fa != SC_SKIP && a == tb;
            }
            const unsigned any = __ballot_sync(0xffffffffu, c);
            if (threadIdx.x % SC_GROUP == 0) chained[i / SC_GROUP] = (any >> (threadIdx.x % 32)) & ((1u << SC_GROUP) - 1);
        }
        __syncthreads();
        if (at >= slot4) continue;
        for (int g = 0; g < count; g += SC_GROUP) {
            if (!chained[g / SC_GROUP]) {
                float4 x[SC_GROUP];
#pragma unroll
                for (int j = 0; j < SC_GROUP; ++j) {
                    const int a = from[g + j];
                    x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (j > 0 && a == from[g + (j > 0 ? j - 1 : 0)]) x[j] = x[j > 0 ? j - 1 : 0];      // a fork reads its source once
                    else if (a >= 0) x[j] = __ldcs(place + (size_t)a * slot4);
                }
#pragma unroll
                for (int j = 0; j < SC_GROUP; ++j)
                    if (from[g + j] != SC_SKIP) __stcs(place + (size_t)to[g + j] * slot4, x[j]);
            } else {
#pragma unroll 1
                for (int j = 0; j < SC_GROUP; ++j) {
                    const int a = from[g + j];
                    if (a != SC_SKIP) place[(size_t)to[g + j] * slot4] = a >= 0 ? place[(size_t)a * slot4] : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
        }
    }
}

}  // namespace

dsla_status launch_state_copy(const dsla_state* st, const int32_t* src, const int32_t* dst, int n, cudaStream_t s) {
    const size_t slot4 = (size_t)st->n_states * st->H * st->d_k * st->d_v / 4;
    const size_t blocks = (slot4 + SC_THREADS - 1) / SC_THREADS;
    if (blocks > 0x7fffffffu) return DSLA_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(SC_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, state_copy_kernel, reinterpret_cast<float4*>(st->data), src, dst, n, st->num_slots, slot4) != cudaSuccess) return DSLA_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? DSLA_OK : DSLA_ERR_CUDA;
}

}  // namespace dsla
