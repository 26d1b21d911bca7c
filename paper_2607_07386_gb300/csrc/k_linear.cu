// Linear layer on the 5th-generation tensor cores (bf16 operands, fp32 accumulation):
//
//   forward   out = residual + act(x W^T + bias), pre = x W^T + bias
//   backward  dp = dout act'(pre);  dx = dp W;  dW = dp^T x;  dbias = column sums of dp
//
// The three products are one kernel, k_linear: D[m, n] = sum_k A(m, k) B(n, k), each operand
// contiguous along k or along its rows (the MMA descriptors take either, so nothing is transposed).
// It is persistent and specialised by warp: one thread streams K-blocks of 64 of both operands
// through a ring of shared memory by TMA, one thread issues the MMAs into one of two TMEM
// accumulators, eight warps take the other accumulator through the epilogue.  Every wait is bounded.  Bound by the
// tensor pipe under the power limit: 32768 x 2048 x 2048 with silu, bias and residual takes 185 us alone (1.49
// PFLOP/s) and 210 to 214 us in a row of calls; dx and dW of it 173 and 164 us alone.  A K-block of a 128 x 256 tile is
// 384 rows of loads, which bounds sizes of a few tiles an SM: 1531 x 5448 x 2056 with gelu takes 57 us.
//
// Every CTA loads both operands of its tiles itself: operands may lie in another GPU's memory (every rank of a run on
// several GPUs loads this library), so no load is shared between CTAs.
//
// Few tiles (a narrow layer over many rows, a batch of tokens being decoded) leave SMs idle, so the
// contraction is split and the fp32 shares are joined, in a fixed order, by k_linear_join, which
// then runs the epilogue.  Up to 16 rows the weights' one trip through memory is all that counts:
// k_linear_skinny reads them with 16-byte loads and keeps the rows of x in shared memory.
#include "gdn_internal.h"
#include "tc_common.cuh"

namespace sdm {

namespace {

using namespace tc;

constexpr int BM = 128, BK = 64;
constexpr int EPI_WARPS = 8;                // two per TMEM lane quarter, each half of the tile's columns
constexpr int LT = 64 + 32 * EPI_WARPS;       // producer, MMA issuer, epilogue
constexpr int SMS = 152;

__host__ __device__ constexpr int stages_of(int bn) { return bn == 256 ? 4 : 6; }
__host__ __device__ constexpr uint32_t stage_bytes(int bn) { return (BM + bn) * 128u; }
__host__ __device__ constexpr uint32_t smem_bytes(int bn) { return 1024u + stage_bytes(bn) * stages_of(bn) + 256u + EPI_WARPS * 512u; }

// Row-major [rows, cols] bf16, box {64 columns, box_rows}, 128-byte swizzle.
bool make_map(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int box_rows) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = map_encoder();
    if (!enc) return false;
    cuuint64_t dim[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    cuuint64_t str[1] = {static_cast<cuuint64_t>(cols) * 2};
    cuuint32_t box[2] = {BK, static_cast<cuuint32_t>(box_rows)};
    cuuint32_t es[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dim, str, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The normal distribution function and, in `pdf`, its density times sqrt(2 pi): Abramowitz and Stegun 7.1.26 on
// x = |z| / sqrt(2), off by at most 7.5e-8 (and the tail by at most its own 0.4% down to -6, where gelu is 6e-9, by 3%
// at -12), from the one exponential that the slope of gelu needs as well (with erff the activation gradient of 8192 x 504
// values took 11.6 us, so 9.8).
__device__ __forceinline__ float normal_cdf(float z, float& pdf) {
    const float x = fabsf(z) * 0.70710678118654752f;
    pdf = __expf(-0.5f * z * z);
    const float t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    const float tail = 0.5f * p * t * pdf;             // 1 - cdf(|z|)
    return z >= 0.f ? 1.f - tail : tail;
}
__device__ __forceinline__ float act_fwd(float z, int act) {
    if (act == SDM_ACT_RELU) return z <= 0.f ? 0.f : z;             // NaN stays
    if (act == SDM_ACT_SILU) return __fdividef(z, 1.f + __expf(-z));     // a few float32 ulps, rounded to bf16 below
    if (act == SDM_ACT_GELU) {
        float pdf;
        return z * normal_cdf(z, pdf);
    }
    return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
    if (act == SDM_ACT_RELU) return z <= 0.f ? 0.f : z > 0.f ? 1.f : z;
    if (act == SDM_ACT_SILU) {
        const float p = __fdividef(1.f, 1.f + __expf(-z));
        return p * (1.f + z * (1.f - p));
    }
    if (act == SDM_ACT_GELU) {
        float pdf;
        const float c = normal_cdf(z, pdf);
        return fmaf(z * pdf, 0.39894228040143268f, c);
    }
    return 1.f;
}

// Eight values of the residual; it may be the output buffer (read by the thread that overwrites it), so
// not through the read-only path.
__device__ __forceinline__ uint4 residual8(const LinearOut& o, int64_t at) {
    return *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(o.residual) + at);
}
// Epilogue of eight neighbouring columns of one row: bias (theirs at `bias`), pre-activation, activation, residual.
__device__ __forceinline__ void finish8(float (&v)[8], const LinearOut& o, int64_t at, const float* bias, const uint4& res) {
    if (o.bias != nullptr) {
        const float4 b0 = *reinterpret_cast<const float4*>(bias), b1 = *reinterpret_cast<const float4*>(bias + 4);
        v[0] += b0.x; v[1] += b0.y; v[2] += b0.z; v[3] += b0.w;
        v[4] += b1.x; v[5] += b1.y; v[6] += b1.z; v[7] += b1.w;
    }
    if (o.pre != nullptr) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(o.pre) + at) = pack16<BF16>(v);
    if (o.act != SDM_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = act_fwd(v[i], o.act);
    }
    if (o.residual != nullptr) {
        float r[8];
        unpack16<BF16>(res, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(o.out) + at) = pack16<BF16>(v);
}

struct LinearGeom {
    int64_t M;
    int N, nkb;               // K-blocks of 64 in the whole contraction
    int ntm, ntn, splits, kbs;  // tiles, splits, K-blocks per split
};

template <int BN, bool AMN, bool BMN>
__global__ void __launch_bounds__(LT, 1) k_linear(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
                                                  const LinearGeom g, const LinearOut o, float* part, int* err) {
    constexpr int S = stages_of(BN);
    constexpr uint32_t STAGE = stage_bytes(BN);
    constexpr uint32_t COLS = 2 * BN < 32 ? 32 : 2 * BN;
    extern __shared__ unsigned char raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t ring = (base + 1023u) & ~1023u;
    const uint32_t bars = ring + STAGE * S;            // full[S], empty[S], acc full[2], acc empty[2], TMEM address
    const uint32_t full = bars, empty = bars + 8 * S, afull = bars + 16 * S, aempty = afull + 16;
    uint32_t* slot = reinterpret_cast<uint32_t*>(raw + (bars - base) + 16 * S + 32);
    float* const bias_sm = reinterpret_cast<float*>(raw + (bars - base) + 256);
    const int tid = threadIdx.x, warp = tid >> 5;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(slot)), "r"(COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    if (tid == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(afull + 8 * s, 1);
            mbar_init(aempty + 8 * s, 32 * EPI_WARPS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = *slot;
    const int items = g.ntm * g.ntn * g.splits;
    bool ok = true;

    if (tid == 0) {                                    // loads
        uint32_t it = 0;
        for (int w = blockIdx.x; w < items && ok; w += gridDim.x) {
            const int sp = w % g.splits, tile = w / g.splits;
            const int m0 = (tile / g.ntn) * BM, n0 = (tile % g.ntn) * BN;
            const int k0 = sp * g.kbs, k1 = k0 + g.kbs < g.nkb ? k0 + g.kbs : g.nkb;
            for (int kb = k0; kb < k1; ++kb, ++it) {
                const int s = it % S;
                if (it >= S && !mbar_wait(empty + 8 * s, ((it / S) - 1) & 1)) { ok = false; break; }
                const uint32_t a = ring + s * STAGE, b = a + BM * 128, bar = full + 8 * s;
                mbar_expect_tx(bar, STAGE);
                if (AMN) {
#pragma unroll
                    for (int j = 0; j < BM / 64; ++j) tma_load_2d(a + j * 8192, &ta, m0 + 64 * j, kb * BK, bar);
                } else {
                    tma_load_2d(a, &ta, kb * BK, m0, bar);
                }
                if (BMN) {
#pragma unroll
                    for (int j = 0; j < BN / 64; ++j) tma_load_2d(b + j * 8192, &tb, n0 + 64 * j, kb * BK, bar);
                } else {
                    tma_load_2d(b, &tb, kb * BK, n0, bar);
                }
            }
        }
        // the copies in flight land before the CTA may end
        for (uint32_t j = it > S ? it - S : 0; j < it; ++j) mbar_wait(full + 8 * (j % S), (j / S) & 1);
    } else if (tid == 32) {                            // MMAs
        const uint32_t idesc = mma_idesc(BN) | (AMN ? MN_A : 0u) | (BMN ? MN_B : 0u);
        uint32_t it = 0, n = 0;
        for (int w = blockIdx.x; w < items && ok; w += gridDim.x, ++n) {
            const int sp = w % g.splits;
            const int k0 = sp * g.kbs, k1 = k0 + g.kbs < g.nkb ? k0 + g.kbs : g.nkb;
            const uint32_t acc = tmem + (n & 1) * BN;
            if (n >= 2 && !mbar_wait(aempty + 8 * (n & 1), ((n >> 1) - 1) & 1)) { ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
            for (int kb = k0; kb < k1; ++kb, ++it) {
                const int s = it % S;
                if (!mbar_wait(full + 8 * s, (it / S) & 1)) { ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                const uint32_t a = ring + s * STAGE, b = a + BM * 128;
#pragma unroll
                for (int kk = 0; kk < BK / 16; ++kk)
                    mma_bf16(acc, AMN ? sw128_mn_desc(a + kk * 2048, 8192) : sw128_desc(a + kk * 32),
                             BMN ? sw128_mn_desc(b + kk * 2048, 8192) : sw128_desc(b + kk * 32), idesc, (kb != k0 || kk != 0) ? 1u : 0u);
                mma_commit(empty + 8 * s);
            }
            if (ok) mma_commit(afull + 8 * (n & 1));
        }
    } else if (warp >= 2) {                            // epilogue: TMEM lanes of this warp's quadrant
        const int quad = warp & 3, part_of = (warp - 2) >> 2, lane = tid & 31;
        uint32_t n = 0;
        for (int w = blockIdx.x; w < items && ok; w += gridDim.x, ++n) {
            const int sp = w % g.splits, tile = w / g.splits;
            const int n0 = (tile % g.ntn) * BN;
            const int64_t row = static_cast<int64_t>(tile / g.ntn) * BM + quad * 32 + lane;
            constexpr int BLOCKS = BN / 64;                // blocks of 32 columns of this warp
            const int c0 = part_of * (BN / 2);
            const uint32_t src = tmem + (n & 1) * BN + c0 + (static_cast<uint32_t>(quad * 32) << 16);
            const bool res = o.residual != nullptr && part == nullptr && row < g.M;
            float* const bias = bias_sm + (warp - 2) * 128;    // this warp's columns
            if (o.bias != nullptr && part == nullptr) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < BN / 64; ++i) {
                    const int col = n0 + c0 + i * 32 + lane;
                    bias[i * 32 + lane] = col < g.N ? __ldg(o.bias + col) : 0.f;
                }
                __syncwarp();
            }
            uint4 r[4], rn[4];                             // the residual, one block ahead
            auto fetch = [&](int cb) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int col = n0 + c0 + cb * 32 + q * 8;
                    rn[q] = res && cb < BLOCKS && col < g.N ? residual8(o, row * g.N + col) : make_uint4(0, 0, 0, 0);
                }
            };
            fetch(0);
            ok = __all_sync(0xffffffffu, mbar_wait(afull + 8 * (n & 1), (n >> 1) & 1));
            if (!ok) break;
            tc_after_sync();
            // rolled: the four blocks unrolled, with an activation inlined 128 times, do not fit the
            // instruction cache (an odd shape with gelu took 57 us for them)
#pragma unroll 1
            for (int cb = 0; cb < BLOCKS; ++cb) {
#pragma unroll
                for (int q = 0; q < 4; ++q) r[q] = rn[q];
                fetch(cb + 1);
                float v[32];
                tmem_ld32(src + cb * 32, v);
                if (cb == BLOCKS - 1) {
                    tc_before_sync();
                    mbar_arrive(aempty + 8 * (n & 1));
                }
                if (row < g.M) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int col = n0 + c0 + cb * 32 + q * 8;
                        if (col < g.N) {                   // N is a multiple of 8
                            float f[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) f[e] = v[q * 8 + e];
                            const int64_t at = row * g.N + col;
                            if (part != nullptr) {
                                float4* dst = reinterpret_cast<float4*>(part + sp * g.M * g.N + at);
                                dst[0] = make_float4(f[0], f[1], f[2], f[3]);
                                dst[1] = make_float4(f[4], f[5], f[6], f[7]);
                            } else {
                                finish8(f, o, at, bias + cb * 32 + q * 8, r[q]);
                            }
                        }
                    }
                }
            }
        }
    }
    if (!ok && (tid == 0 || tid == 32 || (tid & 31) == 0)) flag_error(err, ERR_TIMEOUT);
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(COLS) : "memory");
}

// Sum of the splits' shares, in order, and the epilogue; eight columns per thread.
__global__ void __launch_bounds__(256) k_linear_join(const float* __restrict__ part, int splits, int64_t M, int N, const LinearOut o) {
    const int64_t total = M * N, i = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) * 8;
    if (i >= total) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) {
        const float4* p = reinterpret_cast<const float4*>(part + s * total + i);
        const float4 a = __ldg(p), b = __ldg(p + 1);
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
        v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    const uint4 r = o.residual != nullptr ? residual8(o, i) : make_uint4(0, 0, 0, 0);
    finish8(v, o, i, o.bias + i % N, r);
}

// Up to MR rows of x: a warp owns two rows of W (output columns), its lanes take 16-byte pieces of
// the contraction, eight of them in flight, the first before x is staged in shared memory (KT columns at a
// time).
constexpr int SKINNY_KT = 2048, SKINNY_U = 4;
template <int MR>
__global__ void __launch_bounds__(256) k_linear_skinny(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ W,
                                                       int M, int N, int K, const LinearOut o) {
    extern __shared__ __align__(16) unsigned char raw[];
    __nv_bfloat16* xs = reinterpret_cast<__nv_bfloat16*>(raw);          // [MR][KT]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n0 = (blockIdx.x * 8 + warp) * 2;
    const bool live = n0 < N;                               // N is even
    const __nv_bfloat16* const w0 = W + static_cast<int64_t>(live ? n0 : 0) * K;
    float acc[2][MR];
#pragma unroll
    for (int m = 0; m < MR; ++m) acc[0][m] = acc[1][m] = 0.f;
    uint4 wv[SKINNY_U][2];
    auto fetch = [&](int c) {                               // columns c + 256 u of W
#pragma unroll
        for (int u = 0; u < SKINNY_U; ++u)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                wv[u][j] = live && c + 256 * u < K ? __ldcs(reinterpret_cast<const uint4*>(w0 + static_cast<int64_t>(j) * K + c + 256 * u)) : make_uint4(0, 0, 0, 0);
    };
    fetch(lane * 8);
    for (int k0 = 0; k0 < K; k0 += SKINNY_KT) {
        const int kt = K - k0 < SKINNY_KT ? K - k0 : SKINNY_KT;
        __syncthreads();
        for (int i = threadIdx.x; i < MR * (kt / 8); i += 256) {
            const int m = i / (kt / 8), c = (i % (kt / 8)) * 8;
            *reinterpret_cast<uint4*>(xs + m * SKINNY_KT + c) =
                m < M ? __ldg(reinterpret_cast<const uint4*>(x + static_cast<int64_t>(m) * K + k0 + c)) : make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
        for (int c = lane * 8; c < kt; c += 256 * SKINNY_U) {
            float w[SKINNY_U][2][8];
#pragma unroll
            for (int u = 0; u < SKINNY_U; ++u)
#pragma unroll
                for (int j = 0; j < 2; ++j) unpack16<BF16>(wv[u][j], w[u][j]);
            fetch(k0 + c + 256 * SKINNY_U);
#pragma unroll
            for (int u = 0; u < SKINNY_U; ++u) {
                if (c + 256 * u >= kt) break;
#pragma unroll
                for (int m = 0; m < MR; ++m) {
                    float f[8];
                    unpack16<BF16>(*reinterpret_cast<const uint4*>(xs + m * SKINNY_KT + c + 256 * u), f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        acc[0][m] = fmaf(f[e], w[u][0][e], acc[0][m]);
                        acc[1][m] = fmaf(f[e], w[u][1][e], acc[1][m]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MR; ++m) {
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) {
            acc[0][m] += __shfl_xor_sync(0xffffffffu, acc[0][m], s);
            acc[1][m] += __shfl_xor_sync(0xffffffffu, acc[1][m], s);
        }
    }
    if (!live) return;
#pragma unroll
    for (int m = 0; m < MR; ++m) {
        if (m < M && lane < 2) {
            const int n = n0 + lane;
            const int64_t at = static_cast<int64_t>(m) * N + n;
            float z = lane ? acc[1][m] : acc[0][m];
            if (o.bias != nullptr) z += __ldg(o.bias + n);
            if (o.pre != nullptr) static_cast<__nv_bfloat16*>(o.pre)[at] = __float2bfloat16_rn(z);
            z = act_fwd(z, o.act);
            if (o.residual != nullptr) z += __bfloat162float(static_cast<const __nv_bfloat16*>(o.residual)[at]);
            static_cast<__nv_bfloat16*>(o.out)[at] = __float2bfloat16_rn(z);
        }
    }
}

// dp = dout act'(pre), rounded to bf16 as an operand of the two products, and the column sums of the
// unrounded values: a CTA takes 64 columns x ROWS rows, thread (y, x) eight columns of every 32nd row.
constexpr int DA_ROWS = 256;
__global__ void __launch_bounds__(256) k_linear_dact(const __nv_bfloat16* __restrict__ dout, const __nv_bfloat16* __restrict__ pre,
                                                     int act, int64_t M, int N, __nv_bfloat16* __restrict__ dp,
                                                     float* __restrict__ part) {
    __shared__ float sum[32][64 + 1];
    const int x = threadIdx.x & 7, y = threadIdx.x >> 3;
    const int col = blockIdx.x * 64 + x * 8;
    const int64_t r0 = static_cast<int64_t>(blockIdx.y) * DA_ROWS;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (col < N) {
#pragma unroll
        for (int jj = 0; jj < DA_ROWS / 32; jj += 4) {
            uint4 du[4], zu[4];                            // four rows of loads in flight
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t row = r0 + (jj + j) * 32 + y;
                du[j] = zu[j] = make_uint4(0, 0, 0, 0);
                if (row < M) {
                    du[j] = __ldcs(reinterpret_cast<const uint4*>(dout + row * N + col));
                    if (act != SDM_ACT_NONE) zu[j] = __ldcs(reinterpret_cast<const uint4*>(pre + row * N + col));
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t row = r0 + (jj + j) * 32 + y;
                if (row >= M) break;
                float d[8], z[8];
                unpack16<BF16>(du[j], d);
                if (act != SDM_ACT_NONE) {
                    unpack16<BF16>(zu[j], z);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] *= act_slope(z[e], act);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += d[e];
                if (dp != nullptr) *reinterpret_cast<uint4*>(dp + row * N + col) = pack16<BF16>(d);
            }
        }
    }
    if (part == nullptr) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[y][x * 8 + e] = acc[e];
    __syncthreads();
    if (threadIdx.x < 64 && blockIdx.x * 64 + threadIdx.x < N) {
        float s = 0.f;
        for (int i = 0; i < 32; ++i) s += sum[i][threadIdx.x];
        part[static_cast<int64_t>(blockIdx.y) * N + blockIdx.x * 64 + threadIdx.x] = s;
    }
}
// dbias[n] = sum over the row blocks, eight ranges of them per column.
__global__ void __launch_bounds__(256) k_linear_dbias(const float* __restrict__ part, int blocks, int N, float* __restrict__ dbias) {
    __shared__ float sum[8][32];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, n = blockIdx.x * 32 + x;
    float s = 0.f;
    if (n < N)
        for (int i = y; i < blocks; i += 8) s += __ldg(part + static_cast<int64_t>(i) * N + n);
    sum[y][x] = s;
    __syncthreads();
    if (y == 0 && n < N) {
        for (int i = 1; i < 8; ++i) s += sum[i][x];
        dbias[n] = s;
    }
}

template <int BN, bool AMN, bool BMN>
cudaError_t launch_tiles(const CUtensorMap& ta, const CUtensorMap& tb, const LinearGeom& g, const LinearOut& o, float* part,
                         int* err, cudaStream_t stream) {
    constexpr uint32_t smem = smem_bytes(BN);
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_linear<BN, AMN, BMN>, smem, seen);
    if (e != cudaSuccess) return e;
    const int64_t items = static_cast<int64_t>(g.ntm) * g.ntn * g.splits;
    k_linear<BN, AMN, BMN><<<static_cast<unsigned>(items < SMS ? items : SMS), LT, smem, stream>>>(ta, tb, g, o, part, err);
    return cudaGetLastError();
}

template <int BN>
cudaError_t launch_majors(bool a_mn, bool b_mn, const CUtensorMap& ta, const CUtensorMap& tb, const LinearGeom& g,
                          const LinearOut& o, float* part, int* err, cudaStream_t stream) {
    if (!a_mn && !b_mn) return launch_tiles<BN, false, false>(ta, tb, g, o, part, err, stream);
    if (!a_mn) return launch_tiles<BN, false, true>(ta, tb, g, o, part, err, stream);
    return launch_tiles<BN, true, true>(ta, tb, g, o, part, err, stream);
}

}  // namespace

bool linear_skinny(int64_t M) { return M <= 16; }

// 128 x 256 tiles read least from L2 per product; narrower ones only where fewer than half of the SMs
// would have a tile.  Then the contraction is split until the tiles cover the SMs, each share
// keeping at least 4 K-blocks (256 terms).  Measured at K = 2048: 96 to 128 wide tiles (512 x 6144, 1531 x 2048,
// 1024 x 4096) 18.7 to 20.7 us, in half the width, twice as many, 24.7 to 24.9; 256 x 6144 in 96 tiles of 128 columns 16.5, in
// 192 of 64 22.8; 96 wide tiles in two splits 32 to 41.  At 76 wide tiles, which the rule splits in two, half the width
// would do better (2432 x 1024: 16.4 against 23.1).
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K) {
    const int64_t tm = (M + BM - 1) / BM, nkb = (K + BK - 1) / BK;
    int bn = 256;
    while (bn > 64 && tm * ((N + bn - 1) / bn) * 2 < SMS) bn /= 2;
    const int64_t tiles = tm * ((N + bn - 1) / bn);
    int64_t splits = tiles * 2 <= SMS ? SMS / tiles : 1;
    if (splits > nkb / 4) splits = nkb / 4;
    if (splits > 16) splits = 16;
    if (splits < 1) splits = 1;
    const int64_t kbs = (nkb + splits - 1) / splits;
    return LinearPlan{bn, static_cast<int>((nkb + kbs - 1) / kbs)};
}

size_t linear_split_bytes(int64_t M, int64_t N, int64_t K) {
    const LinearPlan p = linear_plan(M, N, K);
    return p.splits > 1 ? static_cast<size_t>(p.splits) * M * N * 4 : 0;
}

cudaError_t launch_linear(const void* A, bool a_mn, const void* B, bool b_mn, int64_t M, int64_t N, int64_t K,
                          const LinearOut& o, float* split_ws, int* err, cudaStream_t stream) {
    const LinearPlan p = linear_plan(M, N, K);
    CUtensorMap ta, tb;
    if (!(a_mn ? make_map(&ta, A, K, M, BK) : make_map(&ta, A, M, K, BM)) ||
        !(b_mn ? make_map(&tb, B, K, N, BK) : make_map(&tb, B, N, K, p.bn)))
        return cudaErrorInvalidValue;
    LinearGeom g{};
    g.M = M;
    g.N = static_cast<int>(N);
    g.nkb = static_cast<int>((K + BK - 1) / BK);
    g.ntm = static_cast<int>((M + BM - 1) / BM);
    g.ntn = static_cast<int>((N + p.bn - 1) / p.bn);
    g.splits = p.splits;
    g.kbs = (g.nkb + p.splits - 1) / p.splits;
    float* part = p.splits > 1 ? split_ws : nullptr;
    cudaError_t e = p.bn == 256   ? launch_majors<256>(a_mn, b_mn, ta, tb, g, o, part, err, stream)
                    : p.bn == 128 ? launch_majors<128>(a_mn, b_mn, ta, tb, g, o, part, err, stream)
                                  : launch_majors<64>(a_mn, b_mn, ta, tb, g, o, part, err, stream);
    if (e != cudaSuccess || part == nullptr) return e;
    const int64_t pieces = M * N / 8;
    k_linear_join<<<static_cast<unsigned>((pieces + 255) / 256), 256, 0, stream>>>(part, p.splits, M, g.N, o);
    return cudaGetLastError();
}

cudaError_t launch_linear_skinny(const void* x, const void* W, int M, int N, int K, const LinearOut& o, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>((N + 15) / 16);
    static std::atomic<unsigned long long> seen;                // only the widest form needs more than 48 KB
    auto go = [&](auto kern, int mr) {
        const size_t smem = static_cast<size_t>(mr) * SKINNY_KT * 2;
        cudaError_t e = allow_smem(kern, smem, seen);
        if (e != cudaSuccess) return e;
        kern<<<grid, 256, smem, stream>>>(static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(W), M, N, K, o);
        return cudaGetLastError();
    };
    if (M <= 1) return go(k_linear_skinny<1>, 1);
    if (M <= 2) return go(k_linear_skinny<2>, 2);
    if (M <= 4) return go(k_linear_skinny<4>, 4);
    if (M <= 8) return go(k_linear_skinny<8>, 8);
    return go(k_linear_skinny<16>, 16);
}

size_t linear_dact_bytes(int64_t M, int64_t N) { return static_cast<size_t>((M + DA_ROWS - 1) / DA_ROWS) * N * 4; }

cudaError_t launch_linear_dact(const void* dout, const void* pre, int act, int64_t M, int N, void* dp, float* dbias,
                               float* part, cudaStream_t stream) {
    const int64_t blocks = (M + DA_ROWS - 1) / DA_ROWS;
    const dim3 grid(static_cast<unsigned>((N + 63) / 64), static_cast<unsigned>(blocks));
    k_linear_dact<<<grid, 256, 0, stream>>>(static_cast<const __nv_bfloat16*>(dout), static_cast<const __nv_bfloat16*>(pre), act,
                                            M, N, static_cast<__nv_bfloat16*>(dp), dbias ? part : nullptr);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || dbias == nullptr) return e;
    k_linear_dbias<<<static_cast<unsigned>((N + 31) / 32), 256, 0, stream>>>(part, static_cast<int>(blocks), N, dbias);
    return cudaGetLastError();
}

}  // namespace sdm
