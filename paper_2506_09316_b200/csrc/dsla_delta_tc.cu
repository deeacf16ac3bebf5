// Gated delta rule over prompts on the tensor cores (bf16, heads of 64 or 128), in chunks of 64 tokens:
//     S <- g S,   u = beta (v - k S),   S <- S + k^T u,   o = scale q S .
// With L_j the sum of log2 g up to token j of the chunk, G_j = 2^L_j, D_ji = 2^(L_j - L_i) and
//     A = tril(beta_j D_ji k_j.k_i, -1),   T = (I + A)^-1 diag(beta),   P = scale tril(D_ji q_j.k_i),   Y = K^T diag(2^(L_63 - L)) T
// a chunk is
//     R = V - G K S,       O = scale G Q S + (P T) R,       S <- G_63 S + Y R .
// Y and P T need no state: a first kernel computes them for all chunks at once (one CTA per chunk and head) into the workspace, a second one walks the
// chunks of each sequence, two dependent products to a chunk, one CTA per (sequence, head, 32 columns of d_v), or more columns where there are many heads.
//
// Precision.  K, Q, V are bf16 as they come.  What reaches a state or an output is held in two bf16 terms (16 bits of mantissa: S as the operand of K S and Q S, R, Y, P T and
// its factors) or three (what Y is made of), with fp32 sums; (I + A)^-1 is fp32.  The state itself stays in fp32 registers and each chunk adds one tensor-core sum to
// it, with rounding.  So outputs are off by their own rounding and by less than 3e-6 of the size of their summands (P T in one term: 1.6e-3 of it, as much as the rounding; a
// second term for it costs 3 to 4 % of time); states by up to 1.7e-5 of their head's largest value, which is the rounding of Y (a third term would be half as many MMAs and operand bytes again).
#include <cuda.h>

#include "dsla_delta.cuh"
#include "tc_utils.cuh"

namespace dsla {

using namespace tc;

bool encode_tile_map(CUtensorMap* m, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
                     const cuuint32_t* box, CUtensorMapSwizzle swizzle);      // dsla_prefill_summary.cu

namespace {

constexpr int DC = 64;                          // tokens per chunk
constexpr int TILE = DC * 128;                  // bytes of 64 rows of 64 bf16
// A chunk in the workspace: Y's high terms and its low terms, each [d][64] bf16, as the MMAs read them (128-byte swizzle); P T, [64][64] bf16, swizzled alike; then the low terms of P T's
// diagonal, [64] bf16, 128 bytes of nothing, and G, [64] fp32.  P T has nothing above its diagonal, so its low terms fill that half, turned by 180 degrees: row r holds the high terms
// (r, c) where c <= r, and the low terms (63 - r, 63 - c) where c > r.
template <int D>
struct Chunk {
    static constexpr int Y = D * 128, PT = 2 * Y, META = PT + TILE, BYTES = META + 2 * DC * 4;
};

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
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, const void* src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2) : "memory");
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

// Columns c and c + 1, c even, of row j of a triangle, its diagonal included: which halves of the word belong to it.
__device__ __forceinline__ uint32_t triangle_mask(int j, int c) { return j > c ? 0xffffffffu : j == c ? 0xffffu : 0u; }
// N pieces of eight columns, from piece `first` on, of row j of P T out of a chunk in shared memory: high and low terms.
template <int N>
__device__ __forceinline__ void take_pt(const uint8_t* pt, const uint8_t* diagonal, int j, int first, uint32_t (&hi)[4 * N], uint32_t (&lo)[4 * N]) {
    const uint32_t corner = 0x10001u * reinterpret_cast<const uint16_t*>(diagonal)[j];
    const int m = 63 - j;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int piece = first + i;
        const uint4 x = *reinterpret_cast<const uint4*>(pt + j * 128 + ((piece ^ (j & 7)) << 4)), y = *reinterpret_cast<const uint4*>(pt + m * 128 + (((7 - piece) ^ (m & 7)) << 4));
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.w, y.z, y.y, y.x};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t with = triangle_mask(j, 8 * piece + 2 * e), below = triangle_mask(j - 1, 8 * piece + 2 * e), turned = __byte_perm(ys[e], 0u, 0x1032);
            hi[4 * i + e] = xs[e] & with;
            lo[4 * i + e] = (turned & below) | (corner & with & ~below);
        }
    }
}

// A pair of fp32 in bf16, and what that leaves; and in two bf16 terms, high and low.
__device__ __forceinline__ uint64_t take_bf16(uint64_t x, uint32_t& hi) {
    const float2 y = unpair(x);
    hi = pack_bf16(y.x, y.y);
    return add2(x, pair((hi << 16) ^ 0x80000000u, (hi & 0xffff0000u) ^ 0x80000000u));
}
__device__ __forceinline__ void split_pair(uint64_t x, uint32_t& hi, uint32_t& lo) {
    const float2 z = unpair(take_bf16(x, hi));
    lo = pack_bf16(z.x, z.y);
}

#define WAIT(bar, parity) mbar_wait(bar, parity, abortp, p.status)

// ------------------------------------------------------------------------------------------------ Y and P T of every chunk
// Eight warps, two to a lane quadrant (columns 0..31 and 32..63).  [K; Q] K^T is one MMA of 128 rows; quadrants 0, 1 turn its upper half into A, 2, 3 its lower half
// into P.  (I + A)^-1 in fp32, in A's place: the eight diagonal blocks of 8 by substitution, one column per thread, then three times
//     [a 0; b c]^-1 = [a^-1 0; -c^-1 b a^-1 c^-1]
// for pairs of blocks of 8, 16 and 32, as TF32 products of two terms each (22 bits); a warp takes 16 columns, so that the other factor is split into terms half as often.  Then P T and Y are MMAs, one after the other through
// the same tiles: 56 KB and 64 registers a thread keep four CTAs on an SM.  4096 tokens of 32 heads: 54 us (the products of P T's low terms and
// their packing 3 of them; with 75 KB and three CTAs on an SM 4 % longer; 110 us with a substitution over all 64 rows by 64 threads, 2016 steps of the chain each, and T written two bytes at a time).
constexpr int PREP_THREADS = 256;
constexpr int XP = 68;                                          // pitch of A and its inverse in shared memory, floats
constexpr int PREP_A = 0, PREP_SCRATCH = DC * XP * 4;           // behind K and Q; scratch: [32][8] floats of four pairs of warps
constexpr int PREP_T = 0;                                       // the same room later: T in two terms, then two of the three terms of diag(2^(L_63 - L)) T, then P T
constexpr uint32_t COL_P = 64;                                  // P in two terms, 32 columns of tensor memory each; Y's sums later
constexpr int PREP_WORK = PREP_SCRATCH + 4 * 32 * 8 * 4;
static_assert(PREP_WORK >= 2 * TILE && PREP_WORK % 1024 == 0, "two tiles fit where A and the scratch are");

template <int D>
struct Prep {
    static constexpr int KQ = 2 * TILE * (D / 64), W_LO = TILE;      // the third term of the weighted T takes the place of Q's first tile
    static constexpr int META = KQ + PREP_WORK, SMEM = META + 2 * DC * 4 + 1024;
};

template <int D>
__global__ void __launch_bounds__(PREP_THREADS, 4) delta_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q, const DeltaTcParams tp) {
    using L = Prep<D>;
    using Out = Chunk<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full, done;
    __shared__ uint32_t tmem_base;
    __shared__ int abort_flag;
    __shared__ __align__(16) float mhi[DC], mlo[DC], sbeta[DC], sw[DC], sleft[DC / 2];
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);
    uint8_t* work = sm + L::KQ;
    const DeltaParams& p = tp.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abortp = &abort_flag;
    const int h = blockIdx.x % p.H;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int n, t_begin, len, first;
    const int at = blockIdx.x / p.H;
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
    const int ahead = (c + 1 + 448 / p.H) * DC;

    if (tid == 0) {
        mbar_init(&full, 1);
        mbar_init(&done, 1);
        abort_flag = 0;
        fence_barrier_init();
        const int hq = h / p.group;
        mbar_arrive_expect_tx(&full, L::KQ);
        for (int half = 0; half < D / 64; ++half) {      // rows 0..63 K, 64..127 Q
            tma_load_4d(sm + half * 2 * TILE, &map_k, &full, 0, t0, half, hq);
            tma_load_4d(sm + half * 2 * TILE + TILE, &map_q, &full, 0, t0, half, hq);
        }
        if (ahead < len)      // what a CTA some 450 from here will load
            for (int half = 0; half < D / 64; ++half) {
                tma_prefetch_4d(&map_k, 0, t_begin + ahead, half, hq);
                tma_prefetch_4d(&map_q, 0, t_begin + ahead, half, hq);
            }
    }
    if (warp == 1) { tmem_alloc(&tmem_base, 128); tmem_relinquish(); }
    if (warp == 2) {
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
            if (ahead + j < len) {
                const size_t far = (size_t)(t_begin + ahead + j) * p.H + h;
                asm volatile("prefetch.global.L2 [%0];" ::"l"(p.gate + far));
                asm volatile("prefetch.global.L2 [%0];" ::"l"(p.beta + far));
            }
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
        const double last = __shfl_sync(0xffffffffu, total, 31), middle = __shfl_sync(0xffffffffu, total, 15);
        float* meta = reinterpret_cast<float*>(sm + L::META);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * lane + i;
            const float hi = (float)run[i];
            mhi[j] = -hi;      // minus the sums: differences are additions
            mlo[j] = (float)(hi - run[i]);
            sbeta[j] = beta[i];
            sw[j] = ex2((float)(last - run[i]));
            if (j < 32) sleft[j] = ex2((float)(middle - run[i]));
            meta[DC + j] = ex2(hi);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // The walk's CTAs take their tensor memory before they wait for this grid, so they may start only when every CTA here has its own.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tb = tmem_base;
    if (warp == 0 && elect_one()) {
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
    __syncwarp();
    const int quad = warp & 3, part = warp >> 2, row = 32 * quad + lane, j = row & 63, upper = quad & 1;
    const uint32_t row_addr = tb + ((uint32_t)(32 * quad) << 16) + 32 * part;
    float* A = reinterpret_cast<float*>(work + PREP_A);
    const bool is_p = quad >= 2;
    WAIT(&done, 0);
    tc_fence_after();
    if (live < DC)      // rows of K behind the end meet zeros of T in Y: whatever they hold must be finite
        for (int i = live * 8 + tid; i < DC * 8; i += PREP_THREADS)
#pragma unroll
            for (int half = 0; half < D / 64; ++half) *reinterpret_cast<uint4*>(sm + half * 2 * TILE + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    if (upper >= part) {
        const float f = j < live ? (is_p ? p.scale : sbeta[j]) : 0.f, hj = -mhi[j], lj = -mlo[j];
        const float fr = f * ex2((hj + mhi[31]) + (lj + mlo[31]));      // left of a diagonal block of 32: through the sum up to token 31
        const int last = j >= live ? -1 : is_p ? j : j - 1;             // columns up to this one
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int c0 = 32 * part + 16 * half;
            uint32_t r[16];
            uint64_t x[8];
            tmem_ld16(row_addr + 16 * half, r);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                uint64_t e[2];
                if (upper == part) {
                    const ulonglong2 hs = *reinterpret_cast<const ulonglong2*>(mhi + c0 + i), ls = *reinterpret_cast<const ulonglong2*>(mlo + c0 + i);
                    const float2 u = unpair(add2(add2(pair(hj, hj), hs.x), add2(pair(lj, lj), ls.x))), v = unpair(add2(add2(pair(hj, hj), hs.y), add2(pair(lj, lj), ls.y)));
                    e[0] = mul2(pair(f, f), pair(ex2(u.x), ex2(u.y)));
                    e[1] = mul2(pair(f, f), pair(ex2(v.x), ex2(v.y)));
                } else {
                    const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(sleft + c0 + i);
                    e[0] = mul2(pair(fr, fr), l.x);
                    e[1] = mul2(pair(fr, fr), l.y);
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int at = i + 2 * k;
                    const float2 y = unpair(mul2(pair(r[at], r[at + 1]), e[k]));
                    x[at / 2] = pair(c0 + at <= last ? y.x : 0.f, c0 + at + 1 <= last ? y.y : 0.f);
                }
            }
            if (!is_p) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) *reinterpret_cast<ulonglong2*>(A + j * XP + c0 + 2 * i) = make_ulonglong2(x[i], x[i + 1]);
            } else {      // an operand in tensor memory, two terms, beside the products
                uint32_t hi[8], lo[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) split_pair(x[e], hi[e], lo[e]);
                tmem_st8(row_addr - 32 * part + COL_P + c0 / 2, hi);
                tmem_st8(row_addr - 32 * part + COL_P + 32 + c0 / 2, lo);
            }
        }
    } else if (is_p) {
        const uint32_t zero[16] = {};
        tmem_st16(row_addr - 32 * part + COL_P + 16 * part, zero);
        tmem_st16(row_addr - 32 * part + COL_P + 32 + 16 * part, zero);
    }
    if (is_p) tc_wait_st();
    tc_fence_before();
    __syncthreads();
    float* scratch = reinterpret_cast<float*>(work + PREP_SCRATCH) + (warp & 3) * 256;      // [rows][8] of this warp's, or this pair's, columns
    const int fr_ = lane >> 2, fq = lane & 3;
    if (warp < 4) {
        const int b0 = 16 * warp;
        if (lane < 16) {      // two blocks of 8: thread = column
            const int at8 = b0 + (lane & 8), col = lane & 7;
            float4 a[10];      // rows 1 .. 7 left of the diagonal
#pragma unroll
            for (int i = 1; i < 8; ++i) {
                a[i < 5 ? i - 1 : 2 * i - 6] = *reinterpret_cast<const float4*>(A + (at8 + i) * XP + at8);
                if (i >= 5) a[2 * i - 5] = *reinterpret_cast<const float4*>(A + (at8 + i) * XP + at8 + 4);
            }
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float s0 = i == col ? 1.f : 0.f, s1 = 0.f;
                if (i > 0) {
                    const float4 l = a[i < 5 ? i - 1 : 2 * i - 6];
                    s0 = fmaf(-l.x, x[0], s0);
                    if (i > 1) s1 = fmaf(-l.y, x[1], s1);
                    if (i > 2) s0 = fmaf(-l.z, x[2], s0);
                    if (i > 3) s1 = fmaf(-l.w, x[3], s1);
                    if (i > 4) {
                        const float4 u = a[2 * i - 5];
                        s0 = fmaf(-u.x, x[4], s0);
                        if (i > 5) s1 = fmaf(-u.y, x[5], s1);
                        if (i > 6) s0 = fmaf(-u.z, x[6], s0);
                    }
                }
                x[i] = s0 + s1;
            }
            __syncwarp(0xffffu);
#pragma unroll
            for (int i = 0; i < 8; ++i) A[(at8 + i) * XP + at8 + col] = x[i];
        }
        __syncwarp();
        // the pair of them (rows 8..15 of the fragments are whatever lies below)
        float f[1][4];
        products<1, 1, false>(f, A + (b0 + 8) * XP + b0, XP, 1, A + b0 * XP + b0, XP, 1, 0, 0, 1, lane);
        *reinterpret_cast<float2*>(scratch + fr_ * 8 + 2 * fq) = make_float2(-f[0][0], -f[0][1]);
        __syncwarp();
        products<1, 1, false>(f, A + (b0 + 8) * XP + b0 + 8, XP, 1, scratch, 8, 1, 0, 0, 1, lane);
        *reinterpret_cast<float2*>(A + (b0 + 8 + fr_) * XP + b0 + 2 * fq) = make_float2(f[0][0], f[0][1]);
    }
    __syncthreads();
    float* const cells = reinterpret_cast<float*>(work + PREP_SCRATCH) + (warp & 1) * 512;      // two blocks of [rows][8]
    if (warp < 2) {      // pairs of blocks of 16
        const int c0 = 32 * warp, r0 = c0 + 16;
        float f[2][4];
        products<2, 2, false>(f, A + r0 * XP + c0, XP, 1, A + c0 * XP + c0, XP, 1, 8, 0, 2, lane);
#pragma unroll
        for (int n = 0; n < 2; ++n) put_fragment(cells + 256 * n, 8, f[n], -1.f, lane);
        __syncwarp();
        products<2, 2, false>(f, A + r0 * XP + r0, XP, 1, cells, 8, 1, 256, 0, 2, lane);
#pragma unroll
        for (int n = 0; n < 2; ++n) put_fragment(A + r0 * XP + c0 + 8 * n, XP, f[n], 1.f, lane);
    }
    __syncthreads();
    {
        // the pair of blocks of 32: warp = 16 rows and 16 columns
        const int m0 = 16 * (warp >> 1), n0 = 16 * (warp & 1);
        float f[2][4];
        if (warp < 4) {
            products<4, 2, false>(f, A + (32 + m0) * XP, XP, 1, A + n0, XP, 1, 8, n0 / 8, 4, lane);
#pragma unroll
            for (int n = 0; n < 2; ++n) put_fragment(cells + 256 * n + m0 * 8, 8, f[n], -1.f, lane);
        }
        __syncthreads();
        if (warp < 4) {
            products<4, 2, false>(f, A + (32 + m0) * XP + 32, XP, 1, cells, 8, 1, 256, 0, m0 ? 4 : 2, lane);
#pragma unroll
            for (int n = 0; n < 2; ++n) put_fragment(A + (32 + m0) * XP + n0 + 8 * n, XP, f[n], 1.f, lane);
        }
    }
    __syncthreads();
    // T = inverse diag(beta) into tiles, then with its rows weighted; thread = 16 columns of a row
    const int ts = tid & 63, tc0 = 16 * (tid >> 6);      // (a warp's rows of one column group: no bank is asked twice)
    uint8_t* const t_at = work + PREP_T + ts * 128;
    uint32_t w[3][8];
    {
        uint64_t x[8];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(A + ts * XP + tc0 + i), b = *reinterpret_cast<const ulonglong2*>(sbeta + tc0 + i);
            const float2 u = unpair(mul2(y.x, b.x)), v = unpair(mul2(y.y, b.y));
            x[i / 2] = pair(tc0 + i <= ts ? u.x : 0.f, tc0 + i + 1 <= ts ? u.y : 0.f);
            x[i / 2 + 1] = pair(tc0 + i + 2 <= ts ? v.x : 0.f, tc0 + i + 3 <= ts ? v.y : 0.f);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) split_pair(x[4 * i + e], hi[e], lo[e]);
            const int piece = ((tc0 / 8 + i) ^ (ts & 7)) << 4;
            *reinterpret_cast<uint4*>(t_at + piece) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(t_at + TILE + piece) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async_smem();
        __syncthreads();
        if (warp == 0 && elect_one()) {
            tc_fence_after();
            // P T cancels where keys are alike (its rows are differences of P's), so both factors keep two terms.  Lanes 64..127 of the operand are P; the
            // products of the 64 before them are not read.
            constexpr uint32_t ID = idesc_bf16(128, 64, 0, 1);
            const uint32_t tt = smem_u32(work + PREP_T);
#pragma unroll
            for (int k = 2; k >= 0; --k)      // P_lo T_hi, P_hi T_lo, P_hi T_hi
#pragma unroll
                for (int kk = 0; kk < DC / 16; ++kk)
                    mma_ts(tb, tb + COL_P + (k == 2 ? 32 : 0) + 8 * kk, smem_desc_sw128(tt + (k == 1 ? TILE : 0) + kk * 2048, 16, 1024), ID, k < 2 || kk ? 1u : 0u);
            tc_commit(&done);
        }
        __syncwarp();
        const uint64_t weight = pair(sw[ts], sw[ts]);
#pragma unroll
        for (int i = 0; i < 8; ++i) split_pair(take_bf16(mul2(x[i], weight), w[0][i]), w[1][i], w[2][i]);
    }
    WAIT(&done, 1);
    tc_fence_after();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int piece = ((tc0 / 8 + i) ^ (ts & 7)) << 4;
        *reinterpret_cast<uint4*>(t_at + piece) = make_uint4(w[0][4 * i], w[0][4 * i + 1], w[0][4 * i + 2], w[0][4 * i + 3]);
        *reinterpret_cast<uint4*>(t_at + TILE + piece) = make_uint4(w[1][4 * i], w[1][4 * i + 1], w[1][4 * i + 2], w[1][4 * i + 3]);
        *reinterpret_cast<uint4*>(sm + L::W_LO + ts * 128 + piece) = make_uint4(w[2][4 * i], w[2][4 * i + 1], w[2][4 * i + 2], w[2][4 * i + 3]);
    }
    fence_proxy_async_smem();
    __syncthreads();
    if (warp == 0 && elect_one()) {
        tc_fence_after();
        constexpr uint32_t ID = idesc_bf16(128, 64, 1, 1);      // d = 64 has 64 rows, the other half of the product is not read
        const uint32_t kt = smem_u32(sm), wt = smem_u32(work + PREP_T), w2 = smem_u32(sm + L::W_LO);
#pragma unroll
        for (int k = 2; k >= 0; --k)
#pragma unroll
            for (int kk = 0; kk < DC / 16; ++kk)
                mma_ss(tb + 64, smem_desc_sw128(kt + kk * 2048, 2 * TILE, 1024), smem_desc_sw128((k == 2 ? w2 : wt + k * TILE) + kk * 2048, 16, 1024), ID, k < 2 || kk ? 1u : 0u);
        tc_commit(&done);
    }
    __syncwarp();
    uint32_t pt[2][16];      // P T, high and low terms (nothing right of the diagonal's block of 32)
    const bool packs = is_p && upper >= part, on_diagonal = is_p && upper == part;
    if (packs) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t r[16];
            tmem_ld16(row_addr + 16 * half, r);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) split_pair(pair(r[2 * i], r[2 * i + 1]), pt[0][8 * half + i], pt[1][8 * half + i]);
        }
    }
    WAIT(&done, 0);
    tc_fence_after();
    if (packs) {         // into one tile, where T was; the pieces that hold both, those of the diagonal, by way of [64][8] of each behind it
        uint8_t *const tile = work + PREP_T, *const edge = work + 2 * TILE;
        const int mine = j >> 3, m = 63 - j;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int piece = 4 * part + i;
            const uint32_t* l = pt[1] + 4 * i;
            if (piece <= mine) {
                uint8_t* const at = piece < mine ? tile + j * 128 + ((piece ^ (j & 7)) << 4) : edge + j * 16;
                uint8_t* const turned = piece < mine ? tile + m * 128 + (((7 - piece) ^ (m & 7)) << 4) : edge + (DC + j) * 16;
                *reinterpret_cast<uint4*>(at) = make_uint4(pt[0][4 * i], pt[0][4 * i + 1], pt[0][4 * i + 2], pt[0][4 * i + 3]);
                *reinterpret_cast<uint4*>(turned) = make_uint4(__byte_perm(l[3], 0u, 0x1032), __byte_perm(l[2], 0u, 0x1032), __byte_perm(l[1], 0u, 0x1032), __byte_perm(l[0], 0u, 0x1032));
            }
        }
        if (on_diagonal) {
            asm volatile("bar.sync 1, 64;" ::: "memory");      // two warps, a thread to a row
            const uint4 x = *reinterpret_cast<const uint4*>(edge + j * 16), y = *reinterpret_cast<const uint4*>(edge + (DC + m) * 16);
            const int e = j & 7;
            const uint32_t k0 = triangle_mask(e, 0), k1 = triangle_mask(e, 2), k2 = triangle_mask(e, 4), k3 = triangle_mask(e, 6);
            *reinterpret_cast<uint4*>(tile + j * 128 + ((mine ^ e) << 4)) =
                make_uint4((x.x & k0) | (y.x & ~k0), (x.y & k1) | (y.y & ~k1), (x.z & k2) | (y.z & ~k2), (x.w & k3) | (y.w & ~k3));
            reinterpret_cast<uint16_t*>(sm + L::META)[j] = reinterpret_cast<const uint16_t*>(edge + (DC + j) * 16)[7 - e];
        }
    }
    if (row < D) {      // Y where K and Q were
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t r[16];
            tmem_ld16(row_addr + 64 + 16 * half, r);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) split_pair(pair(r[8 * i + 2 * e], r[8 * i + 2 * e + 1]), hi[e], lo[e]);
                const int at16 = row * 128 + (((4 * part + 2 * half + i) ^ (row & 7)) << 4);
                *reinterpret_cast<uint4*>(sm + at16) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4*>(sm + Out::Y + at16) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    if (tid == 0) {
        uint8_t* to = tp.ws + ((size_t)at * p.H + h) * Out::BYTES;
        bulk_store(to, sm, 2 * Out::Y);
        bulk_store(to + Out::PT, work + PREP_T, TILE);
        bulk_store(to + Out::META, sm + L::META, 2 * DC * 4);
        bulk_commit();
        bulk_wait_read();
    }
    settle_after_timeout(abortp);
    if (warp == 1) tmem_dealloc(tb, 128);
}

// ------------------------------------------------------------------------------------------------ the walk over a sequence's chunks
// Warps 0..7 work on rows, two for each lane quadrant (16 columns each), 8 issues the MMAs, 9 loads.  (Issued by a row warp the MMAs hold up that warp's rows: 2750
// cycles per chunk instead of 2450.)  With W = 32 columns of d_v, per chunk:
//   [K; Q] [S_hi | S_lo]          128 x 64 x d    lanes 0..63 K S, 64..127 Q S
//   Y_hi [R_hi | R_lo] + Y_lo R_hi   128 x 64 x 64   lanes d_k; on the chain (low by low left out: 2^-16 at most)
//   PT_hi [R_hi | R_lo] + PT_lo R_hi   the same, lanes 64..127, P T out of tensor memory; behind it
// The state is 16 fp32 registers of each thread (lane = d_k).  Quadrants 0 and 1 make R; 2 and 3 finish the outputs of a chunk while the next one's first product
// runs, and take its P T apart into tensor memory.  K and Q are free as soon as that product is done, Y and P T with the last: the two groups of a stage have barriers of their own.
// Bound by shared memory and the chain: a chunk takes 2360 cycles; copies in (78 KB), operands of 24 MMAs (104 KB) and the rows' own accesses hold its port for most of them.
// Slices of a sequence, the first kernel for one slice under the walk of the slice before, took as long as one after the other (4096 tokens 151 us).
// Where the slabs of 32 columns do not all fit on the device at once, fewer and wider ones do more in all: whole heads for d = 128 (delta_walk_wide_kernel), 64 columns for d = 64
// (32 heads of 64, 64 sequences of 512 tokens: 765 us with W = 32, 571 with W = 64; 80 heads, one sequence of 2048: 135 and 112).  A CTA that is done then takes over a block
// of the grid that has not started, two of them ahead: the next one's loads run under the end of this one's, and barriers and tensor memory are set up once (64 sequences of 64
// tokens, 32 heads of 64: 181 us with a CTA for each, 127 so; of 512 tokens 631 and 571).
constexpr int WC = 16, ST = 2;      // columns of a thread; stages of loads

template <int D_, int W_>
struct Walk {
    using In = Chunk<D_>;
    static constexpr int D = D_, W = W_, PARTS = W / WC;
    static constexpr int ROW_WARPS = 4 * PARTS, THREADS = 32 * (ROW_WARPS + 2);
    static constexpr int KQ = 2 * TILE * (D / 64), V = (In::BYTES + 1023) & ~1023, Y_STAGE = V + DC * W * 2, OFF_Y = ST * KQ;
    // Operands of W columns in two terms: rows of [32 high | 32 low], or a tile of 64 high and one of 64 low columns behind each other.
    static constexpr int S_BYTES = D * 4 * W, R_BYTES = DC * 4 * W, S_LBO = D * 128, R_LBO = TILE;
    static constexpr int OFF_S = OFF_Y + ST * Y_STAGE, OFF_R = OFF_S + S_BYTES, OFF_O = OFF_R + R_BYTES, SMEM = OFF_O + 2 * PARTS * 1024 + 1024;
    static constexpr uint32_t COL_X = 0, COL_D = 2 * W, COL_O = 4 * W, COL_P = 6 * W, COLS = W == 32 ? 256 : 512;      // (P T: 32 columns for each term)
    static constexpr uint32_t Y_BYTES = In::BYTES + DC * W * 2;
};

// A wait on the chain of dependent steps: polls, so the thread goes on as soon as the barrier flips, before it parks.
__device__ __forceinline__ void wait_hot(uint64_t* bar, uint32_t parity, volatile int* abortp, int* status) {
#pragma unroll 1
    for (int i = 0; i < 512; ++i)
        if (mbar_test_wait_t<false>(bar, parity)) return;
    mbar_wait_slow<false>(bar, parity, abortp, status, MBAR_WAIT_LIMIT);
}
#define WAIT_HOT(bar, parity) wait_hot(bar, parity, abortp, p.status)
// Rows to the MMA warp, through named barriers: all row warps (or half of them) arrive, it alone waits.  (Every wait before an arrival is bounded, so each arrives.)
template <int ID, int WARPS>
__device__ __forceinline__ void rows_arrive() { asm volatile("bar.arrive %0, %1;" ::"n"(ID), "n"(32 * (WARPS + 1)) : "memory"); }
template <int ID, int WARPS>
__device__ __forceinline__ void rows_wait() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(32 * (WARPS + 1)) : "memory"); }

// Columns 16 part .. of row r (pairs of fp32) in two bf16 terms into an operand of W columns; `lbo`: bytes between its tiles of 64.
template <int W>
__device__ __forceinline__ void put_split(uint8_t* tile, int lbo, int r, int part, const uint64_t (&x)[WC / 2]) {
    uint8_t* row = tile + r * 128;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_pair(x[4 * i + e], h[e], l[e]);
        const int piece = 2 * part + i;
        *reinterpret_cast<uint4*>(row + ((piece ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(row + (W == 32 ? ((piece + 4) ^ (r & 7)) << 4 : lbo + ((piece ^ (r & 7)) << 4))) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// What a CTA works on: one sequence, head and W columns.  `chunks` < 0: nothing any more.
struct Item {
    int t_begin, len, first, slot, h, column, chunks;
    bool live;      // has a state to write
};
// Asks for the place in the grid of a CTA that has not started, which then never does.  By one thread; the answer, 16 bytes, arrives at the barrier.
__device__ __forceinline__ void ask_for_next(void* to, uint64_t* bar) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    mbar_arrive_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(to)), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ int next_block(const void* from) {      // -1: all have started
    int x;
    asm volatile(
        "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t.reg .b32 a, b, c, d;\n\t"
        "ld.shared.b128 r, [%1];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "mov.b32 a, -1;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {a, b, c, d}, r;\n\t"
        "mov.b32 %0, a;\n\t}"
        : "=r"(x)
        : "r"(smem_u32(from))
        : "memory");
    return x;
}
// Named barriers between the loading warp and all others: item `it` has been published, and read.  (Both sides get to each: their other waits are bounded.)
template <int THREADS> __device__ __forceinline__ void item_wait(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(THREADS) : "memory"); }
template <int THREADS> __device__ __forceinline__ void item_arrive(int id) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(THREADS) : "memory"); }
constexpr int PUBLISHED = 3, READ = 5;

struct WalkShared {
    __align__(16) uint8_t answer[16];
    uint64_t kq_full[ST], kq_empty[ST], y_full[ST], y_empty[ST], x_full, d_full, o_full, answered;
    uint64_t q_full, d2_full;      // a whole head to a CTA: Q S, and the second half of the state's columns
    Item items[2];
    uint8_t order[128];
    uint32_t tmem_base;
    int abort_flag;
};

// Barriers, tensor memory, and the order of the sequences; returns whether there is one.  `y_readers`: warps that arrive when they have read a stage of Y.
template <class L>
__device__ __forceinline__ bool walk_set_up(WalkShared& sh, const DeltaParams& p, int tid, int warp, int y_readers) {
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(&sh.kq_full[i], 1);
            mbar_init(&sh.kq_empty[i], 1);
            mbar_init(&sh.y_full[i], 1);
            mbar_init(&sh.y_empty[i], 1 + y_readers);
        }
        mbar_init(&sh.answered, 1);
        mbar_init(&sh.x_full, 1);
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.d2_full, 1);
        mbar_init(&sh.d_full, 1);
        mbar_init(&sh.o_full, 1);
        sh.abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == L::ROW_WARPS) { tmem_alloc(&sh.tmem_base, L::COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const bool sorted = p.cu_seqlens && p.N > 1 && p.N <= 128;
    if (sorted) {      // the longest sequences first (103K tokens in 14 sequences of 1 to 16K, 32 heads of 128: 2.46 ms in the order given, 2.30 so)
        if (tid < p.N) {
            const int mine = p.cu_seqlens[tid + 1] - p.cu_seqlens[tid];
            int rank = 0, from = p.cu_seqlens[0];
            for (int k = 0; k < p.N; ++k) {
                const int to = p.cu_seqlens[k + 1], other = to - from;
                rank += other > mine || (other == mine && k < tid);
                from = to;
            }
            sh.order[rank] = (uint8_t)tid;
        }
        __syncthreads();
    }
    return sorted;
}

// The loading warp.
template <class L>
__device__ __forceinline__ void walk_load(WalkShared& sh, const CUtensorMap& map_k, const CUtensorMap& map_q, const CUtensorMap& map_v, const CUtensorMap& map_o,
                                          const DeltaTcParams& tp, uint8_t* sm, bool sorted, int lane) {
    using In = typename L::In;
    constexpr bool MORE = L::W > 32;      // slabs of 32 columns are for grids that fit on the device at once
    constexpr int D = L::D, W = L::W, SLABS = D / W;
    const DeltaParams& p = tp.p;
    volatile int* abortp = &sh.abort_flag;
    int block = blockIdx.x, cc = 0;      // cc: chunks of all items so far
    for (int it = 0;; ++it) {
        Item x{};
        x.chunks = -1;
        if (block >= 0) {
            if (MORE && lane == 0) ask_for_next(sh.answer, &sh.answered);
            const int place = block / (SLABS * p.H), n = sorted ? sh.order[place] : place;
            find_sequence(tp, n, x.t_begin, x.len, x.first);
            x.slot = p.slots ? p.slots[n] : n;
            x.h = (block / SLABS) % p.H;
            x.column = block % SLABS * W;
            x.live = x.slot >= 0 && x.slot < p.num_slots && (x.len > 0 || !p.use_initial_state);
            x.chunks = x.live ? (x.len + DC - 1) / DC : 0;
        }
        if (it >= 2) item_wait<L::THREADS>(READ + (it & 1));
        if (lane == 0) sh.items[it & 1] = x;
        __syncwarp();
        item_arrive<L::THREADS>(PUBLISHED + (it & 1));
        if (block < 0) break;
        if (x.live && p.use_initial_state)      // rows of the state, on their way before they are asked for
            for (int i = lane; i < D; i += 32)
                asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p.state + (((size_t)x.slot * p.H + x.h) * D + i) * D + x.column), "n"(W * 4) : "memory");
        if (lane == 0 && x.chunks > 0) {
            if (cc == 0) prefetch_tensormap(&map_o);
            const int hq = x.h / p.group;
            for (int c = 0; c < x.chunks && !*abortp; ++c, ++cc) {
                const int st = cc % ST, t = x.t_begin + c * DC;
                if (cc >= ST) WAIT(&sh.kq_empty[st], (cc / ST - 1) & 1);
                uint8_t* to = sm + st * L::KQ;
                mbar_arrive_expect_tx(&sh.kq_full[st], L::KQ);
                for (int half = 0; half < D / 64; ++half) {
                    tma_load_4d(to + half * 2 * TILE, &map_k, &sh.kq_full[st], 0, t, half, hq);
                    tma_load_4d(to + half * 2 * TILE + TILE, &map_q, &sh.kq_full[st], 0, t, half, hq);
                }
                if (cc >= ST) WAIT(&sh.y_empty[st], (cc / ST - 1) & 1);
                to = sm + L::OFF_Y + st * L::Y_STAGE;
                mbar_arrive_expect_tx(&sh.y_full[st], L::Y_BYTES);
                bulk_load(to, tp.ws + ((size_t)(x.first + c) * p.H + x.h) * In::BYTES, In::BYTES, &sh.y_full[st]);
                for (int col = 0; col < W; col += 64) tma_load_3d(to + L::V + col / 64 * TILE, &map_v, &sh.y_full[st], x.column + col, x.h, t);
            }
        }
        __syncwarp();
        block = -1;
        if (MORE) {
            WAIT(&sh.answered, it & 1);
            block = __shfl_sync(0xffffffffu, *abortp ? -1 : next_block(sh.answer), 0);
        }
    }
}

template <int D, int W>
__global__ void __launch_bounds__(Walk<D, W>::THREADS, 1) delta_walk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q,
                                                                  const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_o, const DeltaTcParams tp) {
    using L = Walk<D, W>;
    using In = Chunk<D>;
    constexpr int MMA_WARP = L::ROW_WARPS, LOAD_WARP = MMA_WARP + 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ WalkShared sh;
    uint64_t *kq_full = sh.kq_full, *kq_empty = sh.kq_empty, *y_full = sh.y_full, *y_empty = sh.y_empty;
    uint64_t &x_full = sh.x_full, &d_full = sh.d_full, &o_full = sh.o_full;
    Item* items = sh.items;
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);
    const DeltaParams& p = tp.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abortp = &sh.abort_flag;
    const bool sorted = walk_set_up<L>(sh, p, tid, warp, L::ROW_WARPS / 2);      // half of the rows read the gates of a stage off the chain
    const uint32_t tb = sh.tmem_base;

    if (warp == LOAD_WARP) {
        walk_load<L>(sh, map_k, map_q, map_v, map_o, tp, sm, sorted, lane);
    } else if (warp == MMA_WARP) {
        const uint32_t base = smem_u32(sm), s_at = base + L::OFF_S, r_at = base + L::OFF_R;
        constexpr uint32_t ID = idesc_bf16(128, 2 * W, 0, 1), ID_HI = idesc_bf16(128, W, 0, 1);
        int c = 0;      // chunks of all items
        for (int it = 0;; ++it) {
            item_wait<L::THREADS>(PUBLISHED + (it & 1));
            const int chunks = items[it & 1].chunks;
            __syncwarp();
            if (chunks < 0) break;
            item_arrive<L::THREADS>(READ + (it & 1));
            for (const int end = c + chunks; c < end; ++c) {
                const int st = c % ST;
                const uint32_t kq = base + st * L::KQ, y = base + L::OFF_Y + st * L::Y_STAGE;
                WAIT(&kq_full[st], (c / ST) & 1);
                rows_wait<1, L::ROW_WARPS>();
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        mma_ss(tb + L::COL_X, smem_desc_sw128(kq + (kk / 4) * 2 * TILE + (kk % 4) * 32, 16, 1024), smem_desc_sw128(s_at + kk * 2048, L::S_LBO, 1024), ID, kk ? 1u : 0u);
                    tc_commit(&x_full);
                    tc_commit(&kq_empty[st]);
                }
                __syncwarp();
                WAIT(&y_full[st], (c / ST) & 1);
                rows_wait<2, L::ROW_WARPS / 2>();
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)      // d = 64: rows 64..127 are what lies behind, their lanes are not read
#pragma unroll
                        for (int kk = 0; kk < DC / 16; ++kk)
                            mma_ss(tb + L::COL_D, smem_desc_sw128(y + k * In::Y + kk * 32, 16, 1024), smem_desc_sw128(r_at + kk * 2048, L::R_LBO, 1024), k ? ID_HI : ID, k || kk ? 1u : 0u);
                    tc_commit(&d_full);
                }
                __syncwarp();
                rows_wait<7, L::ROW_WARPS / 2>();      // P T is there, and the sums of the chunk before have been read
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)      // P T in lanes 64..127; what the lanes before them give is not read
#pragma unroll
                        for (int kk = 0; kk < DC / 16; ++kk)
                            mma_ts(tb + L::COL_O, tb + L::COL_P + 32 * k + 8 * kk, smem_desc_sw128(r_at + kk * 2048, L::R_LBO, 1024), k ? ID_HI : ID, k || kk ? 1u : 0u);
                    tc_commit(&o_full);
                    tc_commit(&y_empty[st]);
                }
                __syncwarp();
            }
        }
    } else {
        const int quad = warp & 3, row = 32 * quad + lane;      // lane of TMEM: d_k of the state; token (quadrants 0, 1: of R, 2, 3: of the outputs)
        const int part = warp >> 2;                             // which 16 of the W columns
        const uint32_t lane_addr = tb + ((uint32_t)(32 * quad) << 16) + WC * part;
        const bool has_state = row < D, makes_r = quad < 2;
        const int j = row & 63;
        uint64_t s[WC / 2], y[WC / 2];
#pragma unroll
        for (int i = 0; i < WC / 2; ++i) y[i] = 0;
        int cc = 0;                                             // chunks of all items so far
        // The outputs of chunk c (quadrants 2, 3), the latest of all: y, scaled, and P T R.  Whole rows of 32 tokens leave by a TMA store of this warp; the stores of a ragged end
        // come from the registers.
        uint8_t* o_tile = sm + L::OFF_O + ((quad & 1) * L::PARTS + part) * 1024;
        auto outputs = [&](const Item& x, int c) {
            uint32_t a[WC], b[WC];
            WAIT_HOT(&o_full, (cc - 1) & 1);
            tc_fence_after();
            tmem_ld16(lane_addr + L::COL_O, a);
            tmem_ld16(lane_addr + L::COL_O + W, b);
            tc_wait_ld();
            tc_fence_before();
            uint32_t z[WC / 2];
#pragma unroll
            for (int i = 0; i < WC / 2; ++i) {
                const float2 u = unpair(add2(y[i], add2(pair(a[2 * i], a[2 * i + 1]), pair(b[2 * i], b[2 * i + 1]))));
                z[i] = pack_bf16(u.x, u.y);
            }
            const int t0 = c * DC + 32 * (quad & 1);      // this warp's first token
            if (t0 + 32 <= x.len) {
                if (lane == 0) bulk_wait_read();
                __syncwarp();
                *reinterpret_cast<uint4*>(o_tile + lane * 32) = make_uint4(z[0], z[1], z[2], z[3]);
                *reinterpret_cast<uint4*>(o_tile + lane * 32 + 16) = make_uint4(z[4], z[5], z[6], z[7]);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    tma_store_3d(&map_o, o_tile, x.column + WC * part, x.h, x.t_begin + t0);
                    bulk_commit();
                }
            } else if (t0 + lane < x.len) {
                uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.o) + ((size_t)(x.t_begin + t0 + lane) * p.H + x.h) * D + x.column + WC * part);
                to[0] = make_uint4(z[0], z[1], z[2], z[3]);
                to[1] = make_uint4(z[4], z[5], z[6], z[7]);
            }
        };
        for (int it = 0;; ++it) {
            item_wait<L::THREADS>(PUBLISHED + (it & 1));
            const Item x = items[it & 1];
            __syncwarp();
            if (x.chunks < 0) break;
            item_arrive<L::THREADS>(READ + (it & 1));
            float* S = p.state + (((size_t)x.slot * p.H + x.h) * D + row) * D + x.column + WC * part;
#pragma unroll
            for (int i = 0; i < WC; i += 4) {
                float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
                if (has_state && x.live && p.use_initial_state) z = *reinterpret_cast<const float4*>(S + i);
                s[i / 2] = pair(z.x, z.y);
                s[i / 2 + 1] = pair(z.z, z.w);
            }
            for (int c = 0; c < x.chunks; ++c, ++cc) {
                const int st = cc % ST, live = min(DC, x.len - c * DC);
                const uint8_t* stage = sm + L::OFF_Y + st * L::Y_STAGE;
                const float* meta = reinterpret_cast<const float*>(stage + In::META);
                uint32_t a[WC], b[WC];
                float last;
                if (has_state) put_split<W>(sm + L::OFF_S, L::S_LBO, row, part, s);
                fence_proxy_async_smem();
                tc_fence_before();
                rows_arrive<1, L::ROW_WARPS>();
                if (makes_r) {
                    WAIT_HOT(&y_full[st], (cc / ST) & 1);
                    last = meta[2 * DC - 1];
                    const float G = -meta[DC + j];
                    uint4 vr[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i)      // rows of 64 or 128 bytes, swizzled
                        vr[i] = *reinterpret_cast<const uint4*>(stage + L::V + j * (W * 2) + (((2 * part + i) ^ (W == 32 ? (j >> 1) & 3 : j & 7)) << 4));
                    WAIT_HOT(&x_full, cc & 1);
                    tc_fence_after();
                    tmem_ld16(lane_addr + L::COL_X, a);
                    tmem_ld16(lane_addr + L::COL_X + W, b);
                    tc_wait_ld();
                    uint64_t r[WC / 2];
#pragma unroll
                    for (int i = 0; i < WC / 2; ++i) {
                        const uint32_t word = reinterpret_cast<const uint32_t*>(vr)[i];
                        r[i] = fma2(pair(G, G), add2(pair(a[2 * i], a[2 * i + 1]), pair(b[2 * i], b[2 * i + 1])), pair(word << 16, word & 0xffff0000u));
                    }
                    if (j >= live) {      // a token behind the sequence's end, whatever it holds
#pragma unroll
                        for (int i = 0; i < WC / 2; ++i) r[i] = 0;
                    }
                    put_split<W>(sm + L::OFF_R, L::R_LBO, j, part, r);
                    fence_proxy_async_smem();
                    tc_fence_before();
                    rows_arrive<2, L::ROW_WARPS / 2>();
                } else {
                    if (c > 0) outputs(x, c - 1);
                    WAIT_HOT(&y_full[st], (cc / ST) & 1);
                    last = meta[2 * DC - 1];
                    const float G = meta[DC + j] * p.scale;
                    {
                        constexpr int WORDS = 32 / L::PARTS;
                        uint32_t hi[WORDS], lo[WORDS];
                        take_pt<WORDS / 4>(stage + In::PT, stage + In::META, j, WORDS / 4 * part, hi, lo);
                        const uint32_t to = tb + ((uint32_t)(32 * quad) << 16) + L::COL_P + WORDS * part;
                        if constexpr (WORDS == 16) {
                            tmem_st16(to, hi);
                            tmem_st16(to + 32, lo);
                        } else {
                            tmem_st8(to, hi);
                            tmem_st8(to + 32, lo);
                        }
                        tc_wait_st();
                        tc_fence_before();
                        rows_arrive<7, L::ROW_WARPS / 2>();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&y_empty[st]);
                    WAIT_HOT(&x_full, cc & 1);
                    tc_fence_after();
                    tmem_ld16(lane_addr + L::COL_X, a);
                    tmem_ld16(lane_addr + L::COL_X + W, b);
                    tc_wait_ld();
#pragma unroll
                    for (int i = 0; i < WC / 2; ++i) y[i] = mul2(pair(G, G), add2(pair(a[2 * i], a[2 * i + 1]), pair(b[2 * i], b[2 * i + 1])));
                }
                WAIT_HOT(&d_full, cc & 1);
                tc_fence_after();
                tmem_ld16(lane_addr + L::COL_D, a);
                tmem_ld16(lane_addr + L::COL_D + W, b);
                tc_wait_ld();
                const uint64_t keep = pair(last, last);
#pragma unroll
                for (int i = 0; i < WC / 2; ++i) s[i] = fma2(keep, s[i], add2(pair(a[2 * i], a[2 * i + 1]), pair(b[2 * i], b[2 * i + 1])));
            }
            if (!makes_r && x.chunks > 0) outputs(x, x.chunks - 1);
            if (has_state && x.live) {
#pragma unroll
                for (int i = 0; i < WC; i += 4) {
                    const float2 u = unpair(s[i / 2]), w = unpair(s[i / 2 + 1]);
                    *reinterpret_cast<float4*>(S + i) = make_float4(u.x, u.y, w.x, w.y);
                }
            }
        }
        if (lane == 0) bulk_wait_read();
    }
    tc_fence_before();
    __syncthreads();
    settle_after_timeout(abortp);
    if (warp == MMA_WARP) tmem_dealloc(tb, L::COLS);
}

// The walk with a whole head of d = 128 to a CTA, everything turned over: lanes of TMEM are columns of d_v.  S^T and R^T are A operands in tensor memory, two terms each, so only
// K, Q, Y and P T, the B operands, pass through shared memory, once for all 128 columns:
//   S^T [K; Q]^T            128 x 128 x 128, two terms    columns 0..63 (K S)^T, 64..127 (Q S)^T
//   R^T Y^T                 128 x 128 x 64, three products of terms (low by low left out: 2^-16 at most); on the chain
//   scale G (Q S)^T + R^T (P T)^T    128 x 64 x 64, three products of terms, onto what the rows put there; behind it
// Sixteen row warps, four to a lane quadrant ("parts"): each has 32 columns of d_k of the state in registers; parts 0 and 1 make R of 32 tokens each, 2 and 3 take P T apart into
// two tiles, scale Q S and finish the outputs of the chunk before.  V comes transposed through ldmatrix in the fragment layout that R is then stored in, outputs leave through stmatrix.
// K S is multiplied ahead of Q S, so that R is made under the latter, and the state's columns in two halves, so that half of them are split into terms under the other half's product.
// Bound by the chain, 4400 cycles a chunk with all that is around it, HBM at 5 TB/s and the tensor pipe 57 % busy (103K ragged tokens, 32 heads, both kernels: 3.15 ms in slabs of 32 columns, 2.30 so; slabs
// of 64 lay half-way; 40 heads, one sequence of 2048 tokens, 40 CTAs instead of 160: 120 us in slabs of 32, 105 so).
struct Wide {
    using In = Chunk<128>;
    static constexpr int D = 128, W = 128, ROW_WARPS = 16, THREADS = 32 * (ROW_WARPS + 2);
    static constexpr int KQ = 4 * TILE, V = (In::BYTES + 1023) & ~1023, Y_STAGE = V + 2 * TILE, OFF_Y = ST * KQ, OFF_PT = OFF_Y + ST * Y_STAGE, OFF_O = OFF_PT + 2 * TILE, SMEM = OFF_O + 8 * 2048 + 1024;
    static constexpr uint32_t COL_SH = 0, COL_SL = 64, COL_RH = 128, COL_RL = 160, COL_O = 192, COL_X = 256, COL_D = 384, COLS = 512;
    static constexpr uint32_t Y_BYTES = In::BYTES + 2 * TILE;
};

__global__ void __launch_bounds__(Wide::THREADS, 1) delta_walk_wide_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q,
                                                                           const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_o, const DeltaTcParams tp) {
    using L = Wide;
    using In = L::In;
    constexpr int D = L::D, MMA_WARP = L::ROW_WARPS, LOAD_WARP = MMA_WARP + 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ WalkShared sh;
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);
    const DeltaParams& p = tp.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abortp = &sh.abort_flag;
    const bool sorted = walk_set_up<L>(sh, p, tid, warp, 0);
    const uint32_t tb = sh.tmem_base;

    if (warp == LOAD_WARP) {
        walk_load<L>(sh, map_k, map_q, map_v, map_o, tp, sm, sorted, lane);
    } else if (warp == MMA_WARP) {
        const uint32_t base = smem_u32(sm);
        constexpr uint32_t ID = idesc_bf16(128, 64, 0, 0);
        // S^T times 64 rows of K or Q, 64 channels of d_k from 16 `from` on, both terms of S.
        auto products = [&](uint32_t rows, int from, uint32_t add, uint32_t to = L::COL_X) {
#pragma unroll
            for (int k = 1; k >= 0; --k)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_ts(tb + to, tb + (k ? L::COL_SL : L::COL_SH) + 8 * (from + kk), smem_desc_sw128(rows + (from / 4) * 2 * TILE + kk * 32, 16, 1024), ID, !k || kk ? 1u : add);
        };
        int c = 0;      // chunks of all items
        for (int it = 0;; ++it) {
            item_wait<L::THREADS>(PUBLISHED + (it & 1));
            const int chunks = sh.items[it & 1].chunks;
            __syncwarp();
            if (chunks < 0) break;
            item_arrive<L::THREADS>(READ + (it & 1));
            for (const int end = c + chunks; c < end; ++c) {
                const int st = c % ST;
                const uint32_t kq = base + st * L::KQ, y = base + L::OFF_Y + st * L::Y_STAGE;
                WAIT(&sh.kq_full[st], (c / ST) & 1);
                rows_wait<1, L::ROW_WARPS / 2>();
                tc_fence_after();
                if (elect_one()) {
                    products(kq, 0, 0);
                }
                __syncwarp();
                rows_wait<8, L::ROW_WARPS / 2>();
                tc_fence_after();
                if (elect_one()) {
                    products(kq, 4, 1);
                    tc_commit(&sh.x_full);
                    products(kq + TILE, 0, 0, L::COL_X + DC);
                    products(kq + TILE, 4, 1, L::COL_X + DC);
                    tc_commit(&sh.q_full);
                    tc_commit(&sh.kq_empty[st]);
                }
                __syncwarp();
                WAIT(&sh.y_full[st], (c / ST) & 1);
                rows_wait<2, L::ROW_WARPS / 2>();
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
#pragma unroll
                        for (int k = 2; k >= 0; --k)      // R_hi Y_lo, R_lo Y_hi, R_hi Y_hi
#pragma unroll
                            for (int kk = 0; kk < DC / 16; ++kk)
                                mma_ts(tb + L::COL_D + 64 * half, tb + (k == 1 ? L::COL_RL : L::COL_RH) + 8 * kk, smem_desc_sw128(y + (k == 2 ? In::Y : 0) + half * TILE + kk * 32, 16, 1024),
                                       ID, k < 2 || kk ? 1u : 0u);
                        tc_commit(half ? &sh.d2_full : &sh.d_full);
                    }
                }
                __syncwarp();
                rows_wait<7, L::ROW_WARPS / 2>();
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 2; k >= 0; --k)      // R_hi PT_lo, R_lo PT_hi, R_hi PT_hi
#pragma unroll
                        for (int kk = 0; kk < DC / 16; ++kk)
                            mma_ts(tb + L::COL_O, tb + (k == 1 ? L::COL_RL : L::COL_RH) + 8 * kk, smem_desc_sw128(base + L::OFF_PT + (k == 2 ? TILE : 0) + kk * 32, 16, 1024), ID, 1u);
                    tc_commit(&sh.o_full);
                    tc_commit(&sh.y_empty[st]);
                }
                __syncwarp();
            }
        }
    } else {
        const int quad = warp & 3, part = warp >> 2, m = lane >> 3;
        const uint32_t lane_addr = tb + ((uint32_t)(32 * quad) << 16);
        const bool makes_r = part < 2;
        const int tok = 32 * (part & 1);      // this warp's tokens of a chunk: R's, or the outputs'
        uint64_t s[16];                       // S^T: columns 32 part .. of d_k
        const uint64_t scale = pair(p.scale, p.scale);
        int cc = 0;                           // chunks of all items so far
        uint8_t* o_tile = sm + L::OFF_O + (quad + 4 * (part & 1)) * 2048;      // 32 tokens x 32 columns, rows of 64 bytes, swizzled
        // The outputs of chunk c (parts 2, 3), the latest of all.  Whole rows of 32 tokens leave by a TMA store of this warp, those of a ragged end row by row.
        auto outputs = [&](const Item& x, int c) {
            uint32_t v[2][16];
            WAIT_HOT(&sh.o_full, (cc - 1) & 1);
            tc_fence_after();
            tmem_ld_16x256b_x4(lane_addr + L::COL_O + tok, v[0]);
            tmem_ld_16x256b_x4(lane_addr + (16u << 16) + L::COL_O + tok, v[1]);
            tc_wait_ld();
            tc_fence_before();
            const int t0 = c * DC + tok;
            if (t0 >= x.len) return;
            if (lane == 0) bulk_wait_read();
            __syncwarp();
            uint32_t z[2][8];
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 8; ++i) z[half][i] = pack_bf16(__uint_as_float(v[half][2 * i]), __uint_as_float(v[half][2 * i + 1]));
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const int r = 8 * (i + (m >> 1)) + (lane & 7);
                    stmatrix_x4_trans(smem_u32(o_tile) + r * 64 + (((2 * half + (m & 1)) ^ ((r >> 1) & 3)) << 4), z[half][2 * i], z[half][2 * i + 1], z[half][2 * i + 2], z[half][2 * i + 3]);
                }
            if (t0 + 32 <= x.len) {
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    tma_store_3d(&map_o, o_tile, 32 * quad, x.h, x.t_begin + t0);
                    bulk_commit();
                }
            } else {
                __syncwarp();
                if (t0 + lane < x.len) {
                    uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.o) + ((size_t)(x.t_begin + t0 + lane) * p.H + x.h) * D + 32 * quad);
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[i] = *reinterpret_cast<const uint4*>(o_tile + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4));
                }
            }
        };
        for (int it = 0;; ++it) {
            item_wait<L::THREADS>(PUBLISHED + (it & 1));
            const Item x = sh.items[it & 1];
            __syncwarp();
            if (x.chunks < 0) break;
            item_arrive<L::THREADS>(READ + (it & 1));
            float* S = p.state + (((size_t)x.slot * p.H + x.h) * D + 32 * part) * D + 32 * quad + lane;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = x.live && p.use_initial_state ? pair(S[2 * i * D], S[(2 * i + 1) * D]) : 0;
            for (int c = 0; c < x.chunks; ++c, ++cc) {
                const int st = cc % ST, live = min(DC, x.len - c * DC);
                const uint8_t* stage = sm + L::OFF_Y + st * L::Y_STAGE;
                const float* meta = reinterpret_cast<const float*>(stage + In::META);
                {
                    uint32_t hi[16], lo[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) split_pair(s[i], hi[i], lo[i]);
                    tmem_st16(lane_addr + L::COL_SH + 16 * part, hi);
                    tmem_st16(lane_addr + L::COL_SL + 16 * part, lo);
                    tc_wait_st();
                }
                tc_fence_before();
                if (makes_r) rows_arrive<1, L::ROW_WARPS / 2>();
                else rows_arrive<8, L::ROW_WARPS / 2>();
                float last;
                if (makes_r) {
                    WAIT_HOT(&sh.y_full[st], (cc / ST) & 1);
                    last = meta[2 * DC - 1];
                    uint64_t G[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 g = *reinterpret_cast<const float2*>(meta + DC + tok + 8 * i + 2 * (lane & 3));
                        G[i] = pair(-g.x, -g.y);
                    }
                    uint32_t vr[2][8];      // V^T in the fragment layout
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const int r = tok + 8 * (i + (m >> 1)) + (lane & 7), piece = 4 * (quad & 1) + 2 * half + (m & 1);
                            ldmatrix_x4_trans(smem_u32(stage) + L::V + (quad >> 1) * TILE + r * 128 + ((piece ^ (r & 7)) << 4), vr[half][2 * i], vr[half][2 * i + 1], vr[half][2 * i + 2],
                                              vr[half][2 * i + 3]);
                        }
                    WAIT_HOT(&sh.x_full, cc & 1);
                    tc_fence_after();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t at = lane_addr + ((uint32_t)(16 * half) << 16);
                        uint32_t a[16];
                        tmem_ld_16x256b_x4(at + L::COL_X + tok, a);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t hi[2], lo[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint32_t word = vr[half][2 * i + e];
                                uint64_t r = fma2(G[i], pair(a[4 * i + 2 * e], a[4 * i + 2 * e + 1]), pair(word << 16, word & 0xffff0000u));
                                if (live < DC) {      // tokens behind the sequence's end, whatever they hold
                                    const int j = tok + 8 * i + 2 * (lane & 3);
                                    const float2 u = unpair(r);
                                    r = pair(j < live ? u.x : 0.f, j + 1 < live ? u.y : 0.f);
                                }
                                split_pair(r, hi[e], lo[e]);
                            }
                            tmem_st_16x128b(at + L::COL_RH + tok / 2 + 4 * i, hi[0], hi[1]);
                            tmem_st_16x128b(at + L::COL_RL + tok / 2 + 4 * i, lo[0], lo[1]);
                        }
                    }
                    tc_wait_st();
                    tc_fence_before();
                    rows_arrive<2, L::ROW_WARPS / 2>();
                } else {
                    if (c > 0) outputs(x, c - 1);
                    WAIT_HOT(&sh.y_full[st], (cc / ST) & 1);
                    last = meta[2 * DC - 1];
                    {      // P T as an operand: a thread has 16 columns of a row
                        const int j = 32 * (quad & 1) + lane, first = 4 * (part & 1) + (quad & 2);
                        uint32_t hi[8], lo[8];
                        take_pt<2>(stage + In::PT, stage + In::META, j, first, hi, lo);
                        uint8_t* const row = sm + L::OFF_PT + j * 128;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int at = ((first + i) ^ (j & 7)) << 4;
                            *reinterpret_cast<uint4*>(row + at) = make_uint4(hi[4 * i], hi[4 * i + 1], hi[4 * i + 2], hi[4 * i + 3]);
                            *reinterpret_cast<uint4*>(row + TILE + at) = make_uint4(lo[4 * i], lo[4 * i + 1], lo[4 * i + 2], lo[4 * i + 3]);
                        }
                        fence_proxy_async_smem();
                    }
                    WAIT_HOT(&sh.q_full, cc & 1);
                    tc_fence_after();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t a[16];
                        tmem_ld16(lane_addr + L::COL_X + DC + tok + 16 * half, a);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const ulonglong2 g = *reinterpret_cast<const ulonglong2*>(meta + DC + tok + 16 * half + i);
                            const float2 u = unpair(mul2(pair(a[i], a[i + 1]), mul2(g.x, scale))), v = unpair(mul2(pair(a[i + 2], a[i + 3]), mul2(g.y, scale)));
                            a[i] = __float_as_uint(u.x);
                            a[i + 1] = __float_as_uint(u.y);
                            a[i + 2] = __float_as_uint(v.x);
                            a[i + 3] = __float_as_uint(v.y);
                        }
                        tmem_st16(lane_addr + L::COL_O + tok + 16 * half, a);
                    }
                    tc_wait_st();
                    tc_fence_before();
                    rows_arrive<7, L::ROW_WARPS / 2>();
                }
                WAIT_HOT(makes_r ? &sh.d_full : &sh.d2_full, cc & 1);
                tc_fence_after();
                const uint64_t keep = pair(last, last);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t a[16];
                    tmem_ld16(lane_addr + L::COL_D + 32 * part + 16 * half, a);
                    tc_wait_ld();
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[8 * half + i] = fma2(keep, s[8 * half + i], pair(a[2 * i], a[2 * i + 1]));
                }
            }
            if (!makes_r && x.chunks > 0) outputs(x, x.chunks - 1);
            if (x.live) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 u = unpair(s[i]);
                    S[2 * i * D] = u.x;
                    S[(2 * i + 1) * D] = u.y;
                }
            }
        }
        if (lane == 0) bulk_wait_read();
    }
    tc_fence_before();
    __syncthreads();
    settle_after_timeout(abortp);
    if (warp == MMA_WARP) tmem_dealloc(tb, L::COLS);
}

// [T_total, H_qk, D] bf16 as (64 elements, t, part of a row, head); a box is 64 tokens of one part, one swizzled tile.
bool make_map(CUtensorMap* m, const void* base, int T_total, int H, int d) {
    cuuint64_t dims[4] = {64, (cuuint64_t)T_total, (cuuint64_t)(d / 64), (cuuint64_t)H};
    cuuint64_t strides[3] = {(cuuint64_t)H * d * 2, 128, (cuuint64_t)d * 2};
    cuuint32_t box[4] = {64, DC, 1, 1};
    return encode_tile_map(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

// [T_total, H, D] bf16 as (element, head, t); a box is `columns` elements of `tokens` tokens.
bool make_slab_map(CUtensorMap* m, const void* base, int T_total, int H, int d, int columns, int tokens, CUtensorMapSwizzle swizzle) {
    cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)H, (cuuint64_t)T_total};
    cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)H * d * 2};
    cuuint32_t box[3] = {(cuuint32_t)columns, 1, (cuuint32_t)tokens};
    return encode_tile_map(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, swizzle);
}

long long chunk_slots(const dsla_delta_prefill_args* a) {
    return a->cu_seqlens ? (long long)a->T_total / DC + a->N : (long long)a->N * ((a->T + DC - 1) / DC);
}

template <class L, class Kernel>
dsla_status launch_walk(cudaLaunchConfig_t& cfg, Kernel kernel, const CUtensorMap& mk, const CUtensorMap& mq, const DeltaTcParams& tp, int T_total) {
    const DeltaParams& p = tp.p;
    const int v_columns = L::W < 64 ? L::W : 64, o_columns = L::W == 128 ? 32 : WC;
    CUtensorMap mv{}, mo{};
    if (T_total > 0 && (!make_slab_map(&mv, p.v, T_total, p.H, L::D, v_columns, DC, v_columns == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B) ||
                        !make_slab_map(&mo, p.o, T_total, p.H, L::D, o_columns, 32, o_columns == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE)))
        return DSLA_ERR_CUDA;
    const long long ctas = (long long)p.N * p.H * (L::D / L::W);
    if (ctas > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM) != cudaSuccess) return DSLA_ERR_CUDA;
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(L::THREADS);
    cfg.dynamicSmemBytes = L::SMEM;
    if (cudaLaunchKernelEx(&cfg, kernel, mk, mq, mv, mo, tp) != cudaSuccess) return DSLA_ERR_CUDA;
    count_launch();
    return DSLA_OK;
}

template <int D>
dsla_status launch(const DeltaTcParams& tp, const dsla_delta_prefill_args* a, cudaStream_t s) {
    const DeltaParams& p = tp.p;
    CUtensorMap mk{}, mq{};
    if (a->T_total > 0 && (!make_map(&mk, p.k, a->T_total, a->H_qk, D) || !make_map(&mq, p.q, a->T_total, a->H_qk, D))) return DSLA_ERR_CUDA;
    const long long prep = a->T_total > 0 ? (long long)tp.slots * p.H : 0;
    if (prep > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(delta_chunk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Prep<D>::SMEM) != cudaSuccess) return DSLA_ERR_CUDA;
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
        cfg.dynamicSmemBytes = Prep<D>::SMEM;
        if (cudaLaunchKernelEx(&cfg, delta_chunk_kernel<D>, mk, mq, tp) != cudaSuccess) return DSLA_ERR_CUDA;
        count_launch();
    } else {
        cfg.numAttrs = 0;      // not ahead of whatever kernel comes before: it may still want tensor memory
    }
    dsla_status rc;
    if ((long long)p.N * p.H * (D / 32) <= sm_count()) rc = launch_walk<Walk<D, 32>>(cfg, delta_walk_kernel<D, 32>, mk, mq, tp, a->T_total);
    else if constexpr (D == 128) rc = launch_walk<Wide>(cfg, delta_walk_wide_kernel, mk, mq, tp, a->T_total);
    else rc = launch_walk<Walk<D, 64>>(cfg, delta_walk_kernel<D, 64>, mk, mq, tp, a->T_total);
    if (rc != DSLA_OK) return rc;
    return cudaGetLastError() == cudaSuccess ? DSLA_OK : DSLA_ERR_CUDA;
}

}  // namespace

size_t delta_tc_workspace_bytes(const dsla_delta_prefill_args* a) {
    return a->T_total > 0 ? (size_t)chunk_slots(a) * a->H * (a->d_k == 128 ? Chunk<128>::BYTES : Chunk<64>::BYTES) : 0;
}

dsla_status launch_delta_tc(const DeltaParams& p, const dsla_delta_prefill_args* a, cudaStream_t s) {
    const long long slots = chunk_slots(a);
    if (slots > 0x7fffffffLL) return DSLA_ERR_UNSUPPORTED;
    DeltaTcParams tp{p, static_cast<uint8_t*>(a->workspace), (a->T + DC - 1) / DC, (int)slots};
    return a->d_k == 128 ? launch<128>(tp, a, s) : launch<64>(tp, a, s);
}

}  // namespace dsla
