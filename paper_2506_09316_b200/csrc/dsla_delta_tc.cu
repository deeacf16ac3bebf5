// Gated delta rule over prompts on the tensor cores (bf16, heads of 64 or 128), in chunks of 64 tokens:
//     S <- g S,   u = beta (v - k S),   S <- S + k^T u,   o = scale q S .
// With L_j the sum of log2 g up to token j of the chunk, G_j = 2^L_j, D_ji = 2^(L_j - L_i) and
//     A = tril(beta_j D_ji k_j.k_i, -1),   T = (I + A)^-1 diag(beta),   P = scale tril(D_ji q_j.k_i),   R = V - G K S ,
// a chunk is       U = T R,       O = scale G Q S + (P T) R,       S <- G_63 S + K^T diag(2^(L_63 - L)) U .
// T and P T need no state: a first kernel computes them for all chunks at once (one CTA per chunk and head) into the workspace, a second one walks the
// chunks of each sequence, three dependent products to a chunk, one CTA per (sequence, head, 32 columns of d_v).
//
// Precision.  K, Q, V are bf16 as they come.  What reaches a state is held in two bf16 terms (16 bits of mantissa: S as the operand of K S, R, T
// below its diagonal, U, both factors of P T) with fp32 sums; T's diagonal, beta, is applied in fp32, where most of U comes from when keys differ.  The state itself stays in fp32
// registers and each chunk adds one tensor-core sum to it, with rounding.  What reaches only the bf16 output (S as the operand of Q S, P T as a factor) has one term.
#include <cuda.h>

#include "dsla_internal.cuh"
#include "tc_utils.cuh"

namespace dsla {

using namespace tc;

bool encode_tile_map(CUtensorMap* m, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
                     const cuuint32_t* box, CUtensorMapSwizzle swizzle);      // dsla_prefill_summary.cu

namespace {

constexpr int DC = 64;                          // tokens per chunk
constexpr int TILE = DC * 128;                  // bytes of 64 rows of 64 bf16
// A chunk in the workspace: T (high terms), P T, T (low terms), each [64][64] bf16 as the MMA reads it (128-byte swizzle), then scale G, G, beta and
// 2^(L_63 - L), each [64] fp32.  T_hi above P T are the 128 rows of one operand.
constexpr int CHUNK_TILES = 3 * TILE, CHUNK_BYTES = CHUNK_TILES + 4 * DC * 4;

struct DeltaTcParams {
    DeltaParams p;
    uint8_t* ws;
    int chunks;         // dense batches: chunks per sequence
    int slots;          // chunk slots of the workspace
};

// Bulk copies between global and shared memory; addresses and sizes are multiples of 16 bytes.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
}

// Sequence n: its tokens and the workspace slot of its first chunk.  A packed sequence from token t on has slots t / 64 + n ..: ceil(len / 64) of them
// never reach the next one's.
__device__ __forceinline__ void find_sequence(const DeltaTcParams& tp, int n, int& t_begin, int& len, int& first) {
    if (tp.p.cu_seqlens) {
        t_begin = tp.p.cu_seqlens[n];
        len = tp.p.cu_seqlens[n + 1] - t_begin;
        first = t_begin / DC + n;
    } else {
        t_begin = n * tp.p.T;
        len = tp.p.T;
        first = n * tp.chunks;
    }
}

// x in two bf16 terms, high and low.
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf16(x, y);
    const float2 h = unpack_bf16(hi);
    lo = pack_bf16(x - h.x, y - h.y);
}

// 32 fp32 values in two bf16 terms into row r of an operand whose rows hold [32 high | 32 low].
__device__ __forceinline__ void put_split(uint8_t* tile, int r, const float (&x)[32]) {
    uint8_t* row = tile + r * 128;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) split2(x[8 * i + 2 * e], x[8 * i + 2 * e + 1], h[e], l[e]);
        *reinterpret_cast<uint4*>(row + ((i ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(row + (((i + 4) ^ (r & 7)) << 4)) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

#define WAIT(bar, parity) mbar_wait(bar, parity, abortp, p.status)

// ------------------------------------------------------------------------------------------------ T and P T of every chunk
// Four warps.  [K; Q] K^T is one MMA of 128 rows; warps 0, 1 turn its upper half into A, warps 2, 3 its lower half into P.  Then 64 threads solve (I + A) T =
// diag(beta), one column each, in fp32: x_i is final at step i and leaves A_ji x_i in every later x_j, so a step's products are independent of each
// other.  P T is a second MMA.  The tiles of K and Q make room for what is made of them.
constexpr int PREP_THREADS = 128;
constexpr int PREP_A = 0;                                   // A transposed, [column][row] fp32; then P's low terms in the second tile
constexpr int PREP_T_HI = 2 * TILE, PREP_P = 3 * TILE, PREP_T_LO = 4 * TILE, PREP_META = 5 * TILE;
constexpr int PREP_SMEM = PREP_META + 4 * DC * 4 + 1024;    // K and Q: from 0 on, 2 tiles (d = 64) or 4

template <int D>
__global__ void __launch_bounds__(PREP_THREADS) delta_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q, const DeltaTcParams tp) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full, done;
    __shared__ uint32_t tmem_base;
    __shared__ int abort_flag;
    __shared__ float lhi[DC], llo[DC], sbeta[DC];
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);
    const DeltaParams& p = tp.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abortp = &abort_flag;
    const int h = blockIdx.x % p.H, at = blockIdx.x / p.H;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int n, t_begin, len, first;
    if (p.cu_seqlens) {      // the last sequence whose slots begin at or before this one
        int lo = 0, hi = p.N - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (p.cu_seqlens[mid] / DC + mid <= at) lo = mid;
            else hi = mid - 1;
        }
        n = lo;
    } else {
        n = at / tp.chunks;
    }
    find_sequence(tp, n, t_begin, len, first);
    const int c = at - first;
    if (c < 0 || c * DC >= len) return;
    const int live = min(DC, len - c * DC), t0 = t_begin + c * DC;

    if (tid == 0) {
        mbar_init(&full, 1);
        mbar_init(&done, 1);
        abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) { tmem_alloc(&tmem_base, 64); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = tmem_base;
    if (tid == 0) {
        const int hq = h / p.group;
        mbar_arrive_expect_tx(&full, 2 * TILE * (D / 64));
        for (int half = 0; half < D / 64; ++half) {      // rows 0..63 K, 64..127 Q
            tma_load_4d(sm + half * 2 * TILE, &map_k, &full, 0, t0, half, hq);
            tma_load_4d(sm + half * 2 * TILE + TILE, &map_q, &full, 0, t0, half, hq);
        }
    }
    if (warp == 1) {
        // sums of logs in fp64, handed on as two floats: differences of neighbours stay exact however far the sum has run
        double run[2];
        float beta[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * lane + i;
            const size_t g = (size_t)(t0 + j) * p.H + h;
            float x = j < live ? p.gate[g] : 1.f;
            x = log2f(x < 0.f ? 0.f : x);
            run[i] = x < -300.f ? -300.f : x;      // a gate of 0: products that contain it are an exact zero
            beta[i] = j < live ? p.beta[g] : 0.f;
        }
        run[1] += run[0];
        double total = run[1];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, total, off);
            if (lane >= off) total += y;
        }
        run[0] += total - run[1];
        run[1] = total;
        const double last = __shfl_sync(0xffffffffu, total, 31);
        float* meta = reinterpret_cast<float*>(sm + PREP_META);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * lane + i;
            const float hi = (float)run[i], G = ex2(hi);
            lhi[j] = hi;
            llo[j] = (float)(run[i] - hi);
            sbeta[j] = beta[i];
            meta[j] = G * p.scale;
            meta[DC + j] = G;
            meta[2 * DC + j] = beta[i];
            meta[3 * DC + j] = ex2((float)(last - run[i]));
        }
    } else if (tid == 0) {
        WAIT(&full, 0);
        tc_fence_after();
        const uint32_t kq = smem_u32(sm);
        constexpr uint32_t ID = idesc_bf16(128, 64, 0, 0);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t a = smem_desc_sw128(kq + (kk / 4) * 2 * TILE + (kk % 4) * 32, 16, 1024);
            mma_ss(tb, a, a, ID, kk ? 1u : 0u);      // B: the first 64 rows of the same tile
        }
        tc_commit(&done);
    }
    __syncthreads();
    WAIT(&done, 0);
    tc_fence_after();
    const int j = tid & 63;
    const uint32_t row_addr = tb + ((uint32_t)(32 * warp) << 16);
    const float hj = lhi[j], lj = llo[j], bj = sbeta[j];
    float* at_ = reinterpret_cast<float*>(sm + PREP_A);
    uint32_t pw[32], pl[32];      // warps 2, 3: row j of P, bf16 pairs, and their low terms
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t r[32];
        tmem_ld32(row_addr + 32 * half, r);
        tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            float x[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int s = 32 * half + i + e;
                x[e] = __uint_as_float(r[i + e]) * ex2((hj - lhi[s]) + (lj - llo[s]));
                if (warp < 2) at_[s * DC + j] = s < j && j < live ? bj * x[e] : 0.f;
                else x[e] = s <= j && j < live ? p.scale * x[e] : 0.f;
            }
            split2(x[0], x[1], pw[16 * half + i / 2], pl[16 * half + i / 2]);
        }
    }
    if (warp >= 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4*>(sm + PREP_P + j * 128 + ((i ^ (j & 7)) << 4)) = make_uint4(pw[4 * i], pw[4 * i + 1], pw[4 * i + 2], pw[4 * i + 3]);
    }
    tc_fence_before();
    __syncthreads();
    if (warp < 2) {
        float x[DC];
#pragma unroll
        for (int i = 0; i < DC; ++i) x[i] = i == j ? bj : 0.f;
#pragma unroll
        for (int s = 0; s < DC - 1; ++s) {
            if (s < 32 && warp == 1) continue;      // columns 32.. begin at row 32
            const float xs = x[s];
#pragma unroll
            for (int i = (s + 1) & ~3; i < DC; i += 4) {
                const float4 a = *reinterpret_cast<const float4*>(at_ + s * DC + i);
                if (i > s) x[i] = fmaf(-a.x, xs, x[i]);
                if (i + 1 > s) x[i + 1] = fmaf(-a.y, xs, x[i + 1]);
                if (i + 2 > s) x[i + 2] = fmaf(-a.z, xs, x[i + 2]);
                if (i + 3 > s) x[i + 3] = fmaf(-a.w, xs, x[i + 3]);
            }
        }
#pragma unroll
        for (int i = 0; i < DC; ++i) {
            const float y = i > j ? x[i] : 0.f;      // below the diagonal
            const __nv_bfloat16 hi = __float2bfloat16_rn(y);
            const uint32_t off = sw128_offset(i, j);
            *reinterpret_cast<__nv_bfloat16*>(sm + PREP_T_HI + off) = hi;
            *reinterpret_cast<__nv_bfloat16*>(sm + PREP_T_LO + off) = __float2bfloat16_rn(y - __bfloat162float(hi));
        }
    }
    __syncthreads();
    if (warp >= 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4*>(sm + PREP_A + TILE + j * 128 + ((i ^ (j & 7)) << 4)) = make_uint4(pl[4 * i], pl[4 * i + 1], pl[4 * i + 2], pl[4 * i + 3]);
    }
    fence_proxy_async_smem();
    __syncthreads();
    if (tid == 0) {
        tc_fence_after();
        // P T cancels where keys are alike (its rows are differences of P's), so both factors keep two terms.  Rows 64..127 of the operands are P; the
        // products of the first 64 are not read.
        const uint32_t p_hi = smem_u32(sm + PREP_T_HI), p_lo = smem_u32(sm + PREP_A), t_hi = smem_u32(sm + PREP_T_HI), t_lo = smem_u32(sm + PREP_T_LO);
        constexpr uint32_t ID = idesc_bf16(128, 64, 0, 1);
#pragma unroll
        for (int kk = 0; kk < DC / 16; ++kk) mma_ss(tb, smem_desc_sw128(p_lo + kk * 32, 16, 1024), smem_desc_sw128(t_hi + kk * 2048, 16, 1024), ID, kk ? 1u : 0u);
#pragma unroll
        for (int kk = 0; kk < DC / 16; ++kk) mma_ss(tb, smem_desc_sw128(p_hi + kk * 32, 16, 1024), smem_desc_sw128(t_lo + kk * 2048, 16, 1024), ID, 1u);
#pragma unroll
        for (int kk = 0; kk < DC / 16; ++kk) mma_ss(tb, smem_desc_sw128(p_hi + kk * 32, 16, 1024), smem_desc_sw128(t_hi + kk * 2048, 16, 1024), ID, 1u);
        tc_commit(&done);
    }
    WAIT(&done, 1);
    tc_fence_after();
    if (warp >= 2) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t r[32];
            tmem_ld32(row_addr + 32 * half, r);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 x = unpack_bf16(pw[16 * half + i]), y = unpack_bf16(pl[16 * half + i]);
                const int s = 32 * half + 2 * i;
                pw[16 * half + i] = pack_bf16(fmaf(x.x + y.x, sbeta[s], __uint_as_float(r[2 * i])), fmaf(x.y + y.y, sbeta[s + 1], __uint_as_float(r[2 * i + 1])));
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4*>(sm + PREP_P + j * 128 + ((i ^ (j & 7)) << 4)) = make_uint4(pw[4 * i], pw[4 * i + 1], pw[4 * i + 2], pw[4 * i + 3]);
        fence_proxy_async_smem();
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0) {
        bulk_store(tp.ws + ((size_t)at * p.H + h) * CHUNK_BYTES, sm + PREP_T_HI, CHUNK_BYTES);
        bulk_commit();
        bulk_wait_all();
    }
    settle_after_timeout(abortp);
    if (warp == 1) tmem_dealloc(tb, 64);
}

// ------------------------------------------------------------------------------------------------ the walk over a sequence's chunks
// Six warps: 0 loads, 1 issues the MMAs, 2..5 are the four lane quadrants.  With W = 32 columns of d_v, per chunk:
//   [K; Q] [S_hi | S_lo]        128 x 64 x d    lanes 0..63 K S, 64..127 Q S
//   [T_hi; P T] [R_hi | R_lo]   128 x 64 x 64   and T_lo R_hi 128 x 32 x 64 beside it
//   K^T [U_hi | U_lo]           128 x 64 x 64   lanes d_k, K as the MN-major operand
// The state is 32 fp32 registers of each thread (lane = d_k).  Quadrants 0 and 1 make R and U, 2 and 3 the outputs meanwhile.
constexpr int WALK_THREADS = 6 * 32, W = 32;
constexpr uint32_t COL_X = 0, COL_U = 64, COL_UL = 128, COL_D = 160, WALK_COLS = 256;

template <int D>
struct Walk {
    static constexpr int KQ = 2 * TILE * (D / 64), STAGE = KQ + ((CHUNK_BYTES + 1023) & ~1023), STAGES = 2;
    static constexpr int OFF_S = STAGES * STAGE, OFF_R = OFF_S + D * 128, OFF_U = OFF_R + TILE, SMEM = OFF_U + TILE + 1024;
    static constexpr uint32_t LOAD_BYTES = KQ + CHUNK_BYTES;
};

template <int D>
__global__ void __launch_bounds__(WALK_THREADS) delta_walk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q, const DeltaTcParams tp) {
    using L = Walk<D>;
    constexpr int SLABS = D / W;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[L::STAGES], empty[L::STAGES], s_ready, r_ready, u_ready, x_full, u_full, d_full;
    __shared__ uint32_t tmem_base;
    __shared__ int abort_flag;
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);
    const DeltaParams& p = tp.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abortp = &abort_flag;
    const int slab = blockIdx.x % SLABS, h = (blockIdx.x / SLABS) % p.H, n = blockIdx.x / (SLABS * p.H);

    if (tid == 0) {
        for (int i = 0; i < L::STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        mbar_init(&s_ready, 4);
        mbar_init(&r_ready, 2);
        mbar_init(&u_ready, 2);
        mbar_init(&x_full, 1);
        mbar_init(&u_full, 1);
        mbar_init(&d_full, 1);
        abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) { tmem_alloc(&tmem_base, WALK_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = tmem_base;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int t_begin, len, first;
    find_sequence(tp, n, t_begin, len, first);
    const int slot = p.slots ? p.slots[n] : n;
    const bool work = slot >= 0 && slot < p.num_slots && (len > 0 || !p.use_initial_state);
    const int nc = work && len > 0 ? (len + DC - 1) / DC : 0;

    if (warp == 0) {
        if (lane == 0) {
            if (nc > 0) { prefetch_tensormap(&map_k); prefetch_tensormap(&map_q); }
            const int hq = h / p.group;
            for (int c = 0; c < nc && !*abortp; ++c) {
                const int st = c % L::STAGES;
                if (c >= L::STAGES) WAIT(&empty[st], (c / L::STAGES - 1) & 1);
                uint8_t* to = sm + st * L::STAGE;
                mbar_arrive_expect_tx(&full[st], L::LOAD_BYTES);
                for (int half = 0; half < D / 64; ++half) {
                    tma_load_4d(to + half * 2 * TILE, &map_k, &full[st], 0, t_begin + c * DC, half, hq);
                    tma_load_4d(to + half * 2 * TILE + TILE, &map_q, &full[st], 0, t_begin + c * DC, half, hq);
                }
                bulk_load(to + L::KQ, tp.ws + ((size_t)(first + c) * p.H + h) * CHUNK_BYTES, CHUNK_BYTES, &full[st]);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t base = smem_u32(sm), s_at = base + L::OFF_S, r_at = base + L::OFF_R, u_at = base + L::OFF_U;
            constexpr uint32_t ID_64 = idesc_bf16(128, 64, 0, 1), ID_32 = idesc_bf16(128, 32, 0, 1), ID_KT = idesc_bf16(128, 64, 1, 1);
            for (int c = 0; c < nc; ++c) {
                const int st = c % L::STAGES;
                const uint32_t kq = base + st * L::STAGE, ch = kq + L::KQ;
                WAIT(&full[st], (c / L::STAGES) & 1);
                WAIT(&s_ready, c & 1);
                tc_fence_after();
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    mma_ss(tb + COL_X, smem_desc_sw128(kq + (kk / 4) * 2 * TILE + (kk % 4) * 32, 16, 1024), smem_desc_sw128(s_at + kk * 2048, 16, 1024), ID_64, kk ? 1u : 0u);
                tc_commit(&x_full);
                WAIT(&r_ready, c & 1);
                tc_fence_after();
#pragma unroll
                for (int kk = 0; kk < DC / 16; ++kk)
                    mma_ss(tb + COL_U, smem_desc_sw128(ch + kk * 32, 16, 1024), smem_desc_sw128(r_at + kk * 2048, 16, 1024), ID_64, kk ? 1u : 0u);
#pragma unroll
                for (int kk = 0; kk < DC / 16; ++kk)      // rows 64..127 are whatever lies behind T_lo: their lanes are not read
                    mma_ss(tb + COL_UL, smem_desc_sw128(ch + 2 * TILE + kk * 32, 16, 1024), smem_desc_sw128(r_at + kk * 2048, 16, 1024), ID_32, kk ? 1u : 0u);
                tc_commit(&u_full);
                WAIT(&u_ready, c & 1);
                tc_fence_after();
#pragma unroll
                for (int kk = 0; kk < DC / 16; ++kk)      // d = 64: lanes 64..127 multiply what lies behind K and Q and are not read
                    mma_ss(tb + COL_D, smem_desc_sw128(kq + kk * 2048, 2 * TILE, 1024), smem_desc_sw128(u_at + kk * 2048, 16, 1024), ID_KT, kk ? 1u : 0u);
                tc_commit(&d_full);
                tc_commit(&empty[st]);
            }
        }
    } else if (work) {
        const int quad = warp & 3, row = 32 * quad + lane;      // lane of TMEM: d_k of the state; token (quadrants 0, 1: of R and U, 2, 3: of the outputs)
        const uint32_t lane_addr = tb + ((uint32_t)(32 * quad) << 16);
        const bool has_state = row < D, first_half = quad < 2;
        const int j = row & 63;
        float* S = p.state + (((size_t)slot * p.H + h) * D + row) * D + slab * W;
        const size_t tok_stride = (size_t)p.H * D;
        const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.v) + ((size_t)t_begin * p.H + h) * D + slab * W;
        __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.o) + ((size_t)t_begin * p.H + h) * D + slab * W;
        float s[W];
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (has_state && p.use_initial_state) x = *reinterpret_cast<const float4*>(S + i);
            s[i] = x.x; s[i + 1] = x.y; s[i + 2] = x.z; s[i + 3] = x.w;
        }
        uint4 vr[4];
        auto fetch_v = [&](int c) {
            const int t = c * DC + j;
#pragma unroll
            for (int i = 0; i < 4; ++i) vr[i] = t < len ? __ldg(reinterpret_cast<const uint4*>(v + (size_t)t * tok_stride) + i) : make_uint4(0u, 0u, 0u, 0u);
        };
        if (first_half && nc > 0) fetch_v(0);
        for (int c = 0; c < nc; ++c) {
            const int st = c % L::STAGES, live = min(DC, len - c * DC);
            const float* meta = reinterpret_cast<const float*>(sm + st * L::STAGE + L::KQ + CHUNK_TILES);
            if (has_state) put_split(sm + L::OFF_S, row, s);
            WAIT(&full[st], (c / L::STAGES) & 1);
            if (live < DC) {
                // rows of K behind the sequence's end meet a U of zero: whatever they hold must be finite
                for (int i = live * 8 + (tid - 64); i < DC * 8; i += 128)
#pragma unroll
                    for (int half = 0; half < D / 64; ++half) *reinterpret_cast<uint4*>(sm + st * L::STAGE + half * 2 * TILE + i * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            // (read ahead of the arrival: nothing of the stage is touched by a warp that the others may have left behind)
            const float G = meta[DC + j], sG = meta[j], last = meta[2 * DC - 1], beta = meta[2 * DC + j], w = meta[3 * DC + j];
            fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_ready);
            if (first_half) {
                float r[W];
                uint32_t a[32];
                WAIT(&x_full, c & 1);
                tc_fence_after();
                tmem_ld32(lane_addr + COL_X, a);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < W; ++i) r[i] = __uint_as_float(a[i]);
                tmem_ld32(lane_addr + COL_X + 32, a);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const uint32_t word = reinterpret_cast<const uint32_t*>(vr)[i / 2];
                    const float x = __uint_as_float(i & 1 ? word & 0xffff0000u : word << 16);
                    r[i] = j < live ? fmaf(-G, r[i] + __uint_as_float(a[i]), x) : 0.f;
                }
                put_split(sm + L::OFF_R, j, r);
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&r_ready);
                if (c + 1 < nc) fetch_v(c + 1);
                WAIT(&u_full, c & 1);
                tc_fence_after();
                tmem_ld32(lane_addr + COL_UL, a);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < W; ++i) r[i] = fmaf(beta, r[i], __uint_as_float(a[i]));
                tmem_ld32(lane_addr + COL_U + 32, a);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < W; ++i) r[i] += __uint_as_float(a[i]);
                tmem_ld32(lane_addr + COL_U, a);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < W; ++i) r[i] = w * (r[i] + __uint_as_float(a[i]));
                put_split(sm + L::OFF_U, j, r);
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&u_ready);
            } else {
                float y[W];
                uint32_t a[32];
                WAIT(&x_full, c & 1);
                tc_fence_after();
                tmem_ld32(lane_addr + COL_X, a);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < W; ++i) y[i] = sG * __uint_as_float(a[i]);
                WAIT(&u_full, c & 1);
                tc_fence_after();
                tmem_ld32(lane_addr + COL_U, a);
                tc_wait_ld();
                const int t = c * DC + j;
                if (j < live) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t x[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[e] = pack_bf16(y[8 * i + 2 * e] + __uint_as_float(a[8 * i + 2 * e]), y[8 * i + 2 * e + 1] + __uint_as_float(a[8 * i + 2 * e + 1]));
                        *(reinterpret_cast<uint4*>(o + (size_t)t * tok_stride) + i) = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                }
            }
            WAIT(&d_full, c & 1);
            tc_fence_after();
            {
                uint32_t a[32];
                tmem_ld32(lane_addr + COL_D + 32, a);
                tc_wait_ld();
                float low[W];
#pragma unroll
                for (int i = 0; i < W; ++i) low[i] = __uint_as_float(a[i]);
                tmem_ld32(lane_addr + COL_D, a);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < W; ++i) s[i] = fmaf(last, s[i], low[i] + __uint_as_float(a[i]));
            }
        }
        if (has_state) {
#pragma unroll
            for (int i = 0; i < W; i += 4) *reinterpret_cast<float4*>(S + i) = make_float4(s[i], s[i + 1], s[i + 2], s[i + 3]);
        }
    }
    tc_fence_before();
    __syncthreads();
    settle_after_timeout(abortp);
    if (warp == 1) tmem_dealloc(tb, WALK_COLS);
}

// [T_total, H_qk, D] bf16 as (64 elements, t, part of a row, head); a box is 64 tokens of one part, one swizzled tile.
bool make_map(CUtensorMap* m, const void* base, int T_total, int H, int d) {
    cuuint64_t dims[4] = {64, (cuuint64_t)T_total, (cuuint64_t)(d / 64), (cuuint64_t)H};
    cuuint64_t strides[3] = {(cuuint64_t)H * d * 2, 128, (cuuint64_t)d * 2};
    cuuint32_t box[4] = {64, DC, 1, 1};
    return encode_tile_map(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

long long chunk_slots(const dsla_delta_prefill_args* a) {
    return a->cu_seqlens ? (long long)a->T_total / DC + a->N : (long long)a->N * ((a->T + DC - 1) / DC);
}

template <int D>
dsla_status launch(const DeltaTcParams& tp, const dsla_delta_prefill_args* a, cudaStream_t s) {
    const DeltaParams& p = tp.p;
    CUtensorMap mk{}, mq{};
    if (a->T_total > 0 && (!make_map(&mk, p.k, a->T_total, a->H_qk, D) || !make_map(&mq, p.q, a->T_total, a->H_qk, D))) return DSLA_ERR_CUDA;
    const long long prep = a->T_total > 0 ? (long long)tp.slots * p.H : 0, walk = (long long)p.N * p.H * (D / W);
    if (prep > 0x7fffffffLL || walk > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(delta_chunk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, PREP_SMEM) != cudaSuccess ||
        cudaFuncSetAttribute(delta_walk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Walk<D>::SMEM) != cudaSuccess)
        return DSLA_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (prep > 0) {
        cfg.gridDim = dim3((unsigned)prep);
        cfg.blockDim = dim3(PREP_THREADS);
        cfg.dynamicSmemBytes = PREP_SMEM;
        if (cudaLaunchKernelEx(&cfg, delta_chunk_kernel<D>, mk, mq, tp) != cudaSuccess) return DSLA_ERR_CUDA;
        count_launch();
    }
    cfg.gridDim = dim3((unsigned)walk);
    cfg.blockDim = dim3(WALK_THREADS);
    cfg.dynamicSmemBytes = Walk<D>::SMEM;
    if (cudaLaunchKernelEx(&cfg, delta_walk_kernel<D>, mk, mq, tp) != cudaSuccess) return DSLA_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? DSLA_OK : DSLA_ERR_CUDA;
}

}  // namespace

size_t delta_tc_workspace_bytes(const dsla_delta_prefill_args* a) { return a->T_total > 0 ? (size_t)chunk_slots(a) * a->H * CHUNK_BYTES : 0; }

dsla_status launch_delta_tc(const DeltaParams& p, const dsla_delta_prefill_args* a, cudaStream_t s) {
    const long long slots = chunk_slots(a);
    if (slots > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    DeltaTcParams tp{p, static_cast<uint8_t*>(a->workspace), (a->T + DC - 1) / DC, (int)slots};
    return a->d_k == 128 ? launch<128>(tp, a, s) : launch<64>(tp, a, s);
}

}  // namespace dsla
