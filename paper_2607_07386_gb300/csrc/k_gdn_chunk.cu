// Gated delta rule in chunks of 64 tokens on the 5th-generation tensor cores (bf16 storage, d_k <= 128).
//
// With the decay products of a chunk, G_ij = prod_{j < l <= i} alpha_l, g_i = prod_{l <= i} alpha_l and
// h_j = prod_{l > j} alpha_l, and the state S before it,
//   L_ij = beta_i G_ij k_i.k_j (j < i),  Z = (I + L)^-1,  P_ij = G_ij q_i.k_j (j <= i),
//   w = Z (beta (v - g K S)),   y = scale (g Q S + P w),   S' = h_0.. : g_63 S + K^T (h w).
// k_gdn_factors computes Z, P and the gate products of every chunk at once; k_gdn_scan then walks the
// chunks of one (sequence, head, 128 columns of the state).  The products G are products of gates,
// never quotients or exponentials of sums, so a gate of zero is exact.
//
// Precision: the state and every sum are fp32.  k and q are exact operands.  What the state depends on
// and is not a bf16 number (S itself, Z, the two stages of w) enters the MMAs as bf16 parts, upper and
// lower (16 significant bits, products of two lower parts left out, about 1e-6); y alone takes P rounded
// to bf16 once, as y is.
#include "gdn_internal.h"
#include "tc_common.cuh"

#include <cuda.h>
#include <cudaTypedefs.h>
#include <type_traits>

namespace sdm {

namespace {

using namespace tc;

constexpr int C = GDN_C64;
constexpr uint32_t MAT = C * C * 2;          // bytes of one [64][64] bf16 matrix
constexpr uint32_t GATES = 3 * C * 4;

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = []() -> PFN_cuTensorMapEncodeTiled_v12000 {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
        return nullptr;
    }();
    return fn;
}

// [B, heads, T, d] or [B, T, heads, d] bf16 as {d, T, heads, B}, boxes of 64 values x 64 tokens.
bool token_map(CUtensorMap* m, const void* base, int token_major, int B, int heads, int T, int d) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t row = static_cast<cuuint64_t>(d) * 2, uT = T, uH = heads;
    cuuint64_t dim[4] = {static_cast<cuuint64_t>(d), uT, uH, static_cast<cuuint64_t>(B)};
    cuuint64_t str[3] = {token_major ? row * uH : row, token_major ? row : row * uT, row * uH * uT};
    cuuint32_t box[4] = {64, C, 1, 1}, es[4] = {1, 1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dim, str, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The chunks' matrices as one [chunks * 3 * 64][64] matrix, boxes of one of them.
bool mat_map(CUtensorMap* m, const void* base, int64_t mats) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dim[2] = {C, static_cast<cuuint64_t>(mats) * C};
    cuuint64_t str[1] = {C * 2};
    cuuint32_t box[2] = {C, C}, es[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dim, str, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ------------------------------------------------------------------------------------------
// Factors of a chunk: one CTA of 128 threads.  One MMA chain gives [K; Q] K^T (128 x 64); thread r
// takes row r of it (k_i.k_j for r < 64, q_i.k_j above) and multiplies it by G along the row.  The
// inverse is a column per thread, eliminated left to right in registers: 2016 fused multiply-adds
// whose factors are shared-memory broadcasts.
// ------------------------------------------------------------------------------------------
constexpr int FT = 128;
constexpr int LP = C + 4;
struct FactorSmem {
    float Lt[C][LP];                          // L transposed; then the inverse's two bf16 parts
    float al[C], be[C];
    unsigned long long bar[2];
    uint32_t tmem;
    int dead;
};
template <int DK>
constexpr size_t factor_smem() { return 1024 + 128 * 2 * DK + sizeof(FactorSmem); }

template <int DK>
__global__ void __launch_bounds__(FT) k_gdn_factors(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tq,
                                                    const GdnArgs a, const GdnFactors f) {
    extern __shared__ unsigned char raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t tile = (base + 1023u) & ~1023u;        // per 64 values of d_k: 64 rows of K, 64 of Q
    FactorSmem& sm = *reinterpret_cast<FactorSmem*>(raw + (tile - base) + 128 * 2 * DK);
    const int tid = threadIdx.x, warp = tid >> 5;
    const int b = blockIdx.z, h = blockIdx.y, ch = blockIdx.x, t0 = ch * C;
    const int hk = h / (a.H / a.Hk);
    const int len = gdn_length(a, b);
    if (t0 >= len) return;
    const int n = len - t0 < C ? len - t0 : C;
    const int64_t chain = static_cast<int64_t>(b) * a.H + h, cid = chain * gridDim.x + ch;
    const uint32_t bar = smem_u32(&sm.bar[0]), done = smem_u32(&sm.bar[1]);

    if (tid == 0) {
        sm.dead = 0;
        mbar_init(bar, 1);
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
    }
    if (warp == 0) tmem_alloc(smem_u32(&sm.tmem), 64);
    if (tid < C) {
        sm.al[tid] = tid < n ? load_elem<BF16>(a.alpha, chain * a.T + t0 + tid) : 1.f;
        sm.be[tid] = tid < n ? load_elem<BF16>(a.beta, chain * a.T + t0 + tid) : 0.f;
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = sm.tmem;
    if (tid == 0) {
        mbar_expect_tx(bar, 128 * 2 * DK);
#pragma unroll
        for (int x = 0; x < DK / 64; ++x) {
            tma_load_4d(tile + x * 16384, &tk, 64 * x, t0, hk, b, bar);
            tma_load_4d(tile + x * 16384 + 8192, &tq, 64 * x, t0, hk, b, bar);
        }
        mbar_wait_or_dead(bar, 0, &sm.dead);
        tc_after_sync();
        const uint32_t idesc = mma_idesc(64);
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            const uint32_t at = tile + (kk / 4) * 16384 + (kk % 4) * 32;
            mma_bf16(tmem, sw128_desc(at), sw128_desc(at), idesc, kk != 0);
        }
        mma_commit(done);
    }
    // row i of the decay products, from the diagonal to the left: G_ii = 1, G_i,j-1 = G_ij alpha_j
    const int i = tid & 63;
    const bool isk = tid < C;
    __syncwarp();
    mbar_wait_or_dead(done, 0, &sm.dead);
    __syncwarp();
    tc_after_sync();
    float x[C];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        float v[32];
        tmem_ld32(tmem + (static_cast<uint32_t>(warp * 32) << 16) + 32 * c, v);
#pragma unroll
        for (int j = 0; j < 32; ++j) x[32 * c + j] = v[j];
    }
    const bool row_on = i < n;
    float G = 1.f;
    const float be = sm.be[i];
#pragma unroll
    for (int j = C - 1; j >= 0; --j) {
        const bool in = row_on && (isk ? j < i : j <= i);
        x[j] = in ? G * (isk ? be * x[j] : x[j]) : 0.f;
        if (isk && i == C - 1) f.gates[cid * 3 * C + 2 * C + j] = G;          // h_j
        if (j <= i) G *= sm.al[j];
    }
    if (isk) {
        f.gates[cid * 3 * C + i] = G;                                         // g_i: all factors up to i
        f.gates[cid * 3 * C + C + i] = be;
#pragma unroll
        for (int j = 0; j < C; ++j) sm.Lt[j][i] = x[j];
    } else {
        uint4* dst = reinterpret_cast<uint4*>(static_cast<char*>(f.mat) + (cid * 3 + 2) * MAT + i * C * 2);
#pragma unroll
        for (int j = 0; j < C / 8; ++j) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = x[8 * j + e];
            dst[j] = pack16<BF16>(v);
        }
    }
    __syncthreads();
    if (isk) {
        const int c = tid;
#pragma unroll
        for (int j = 0; j < C; ++j) x[j] = j == c ? 1.f : 0.f;
        // columns 32.. start at row 32: what is above is zero
        auto eliminate = [&](auto from, auto to) {
#pragma unroll
            for (int j = decltype(from)::value; j < decltype(to)::value; ++j) {
#pragma unroll
                for (int q = (j + 1) / 4; q < C / 4; ++q) {
                    const float4 l = *reinterpret_cast<const float4*>(&sm.Lt[j][4 * q]);
                    if (4 * q > j) x[4 * q] = fmaf(-l.x, x[j], x[4 * q]);
                    if (4 * q + 1 > j) x[4 * q + 1] = fmaf(-l.y, x[j], x[4 * q + 1]);
                    if (4 * q + 2 > j) x[4 * q + 2] = fmaf(-l.z, x[j], x[4 * q + 2]);
                    x[4 * q + 3] = fmaf(-l.w, x[j], x[4 * q + 3]);
                }
            }
        };
        if (warp == 0) eliminate(std::integral_constant<int, 0>{}, std::integral_constant<int, 32>{});
        eliminate(std::integral_constant<int, 32>{}, std::integral_constant<int, C - 1>{});
    }
    __syncthreads();
    uint32_t* z = reinterpret_cast<uint32_t*>(&sm.Lt[0][0]);                  // [64][65] words: upper | lower << 16
    if (isk) {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const __nv_bfloat16 hi = __float2bfloat16_rn(x[j]);
            const __nv_bfloat16 lo = __float2bfloat16_rn(x[j] - __bfloat162float(hi));
            z[j * (C + 1) + tid] = static_cast<uint32_t>(__bfloat16_as_ushort(hi)) | (static_cast<uint32_t>(__bfloat16_as_ushort(lo)) << 16);
        }
    }
    __syncthreads();
    for (int p = tid; p < C * C / 8; p += FT) {
        const int r = p / (C / 8), c = (p % (C / 8)) * 8;
        uint32_t w[8], hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = z[r * (C + 1) + c + e];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            hi[e] = (w[2 * e] & 0xffffu) | (w[2 * e + 1] << 16);
            lo[e] = (w[2 * e] >> 16) | (w[2 * e + 1] & 0xffff0000u);
        }
        char* dst = static_cast<char*>(f.mat) + cid * 3 * MAT + p * 16;
        *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(dst + MAT) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    if (tid == 0 && sm.dead) flag_error(a.err, ERR_TIMEOUT);
    tc_before_sync();
    __syncthreads();
    if (warp == 0) tmem_free(tmem, 64);
}

// ------------------------------------------------------------------------------------------
// The walk over the chunks.  A CTA owns 128 columns of one state; everything is transposed, so that a
// TMEM lane is a column: S^T [columns, d_k], w^T [columns, tokens] are A operands written to TMEM from
// registers, and K, Q, Z, P are B operands as TMA leaves them in shared memory (K twice: along d_k for
// K S, along the tokens for the update).  Per chunk:
//   1  U = S^T K^T, then S^T Q^T                      (MMA; the second runs under step 2)
//   2  R = beta (v - g U)                             (registers, bf16 parts to TMEM)
//   3  w = R Z^T                                      (MMA; g Q S is taken out meanwhile)
//   4  w, h w                                         (registers, bf16 parts to TMEM)
//   5  h w K, then w P^T                              (MMA)
//   6  S = g_63 S + ..                                (registers, bf16 parts to TMEM)
// and the output of a chunk is added up and stored under step 1 of the next.  Two warps share a lane
// quarter: in steps 2 and 4 each takes 32 tokens, in step 6 half of d_k.
//
// The chain of six stages is what bounds it: the tensor pipe is busy for about a third of a chunk.
// ------------------------------------------------------------------------------------------
constexpr int SW = 8;                          // compute warps
constexpr int ST = 32 * SW;
constexpr int NS = 2;                          // bf16 parts of a split operand
// TMEM columns
constexpr uint32_t X_COL = 0, Y_COL = 128, S_COL = 192, R_COL = S_COL + 64 * NS, W_COL = R_COL + 32 * NS, T_COLS = 512;
static_assert(W_COL + 32 * NS <= T_COLS, "TMEM columns");

template <int DK>
struct ScanTile {
    static constexpr uint32_t KQ = 0, V = 128 * 2 * DK, M = V + C * 256, G = M + 3 * MAT, BYTES = G + 1024;
    static constexpr uint32_t LOAD = G + GATES;
    static constexpr int STAGES = 3;
};
struct ScanCtl {
    unsigned long long full[3], step[5];
    uint32_t tmem;
    int dead;
};
template <int DK>
constexpr size_t scan_smem() { return 1024 + ScanTile<DK>::BYTES * ScanTile<DK>::STAGES + sizeof(ScanCtl); }

// 32 values as bf16 parts, 16 packed columns each, `stride` columns apart.
__device__ __forceinline__ void put_parts(uint32_t taddr, uint32_t stride, float (&v)[32]) {
#pragma unroll
    for (int p = 0; p < NS; ++p) {
        uint32_t u[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) u[j] = split2(v[2 * j], v[2 * j + 1], v[2 * j], v[2 * j + 1]);
        tmem_st16(taddr + p * stride, u);
    }
}

template <int DK>
__global__ void __launch_bounds__(ST, 1) k_gdn_scan(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tq,
                                                    const __grid_constant__ CUtensorMap tv, const __grid_constant__ CUtensorMap tm,
                                                    const GdnScan r, const GdnFactors f, int nc) {
    using L = ScanTile<DK>;
    extern __shared__ unsigned char raw[];
    const GdnArgs& a = r.a;
    const uint32_t base = smem_u32(raw);
    const uint32_t ring = (base + 1023u) & ~1023u;
    ScanCtl& ctl = *reinterpret_cast<ScanCtl*>(raw + (ring - base) + L::BYTES * L::STAGES);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b = blockIdx.z, h = blockIdx.y, col0 = blockIdx.x * 128, hk = h / (a.H / a.Hk);
    const int len = gdn_length(a, b);
    const int64_t chain = static_cast<int64_t>(b) * a.H + h;
    const int chunks = (len + C - 1) / C;
    const uint32_t full = smem_u32(&ctl.full[0]), step = smem_u32(&ctl.step[0]);
    if (tid == 0) {
        ctl.dead = 0;
        for (int s = 0; s < L::STAGES; ++s) mbar_init(full + 8 * s, 1);
        for (int s = 0; s < 5; ++s) mbar_init(step + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
    }
    if (warp == 0) tmem_alloc(smem_u32(&ctl.tmem), T_COLS);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = ctl.tmem;
    volatile int* dead = &ctl.dead;

    // chunk tiles, by thread 32; a stage is filled again once step 5 of its last chunk is through
    auto load = [&](int c) {
        const uint32_t t = ring + (c % L::STAGES) * L::BYTES, bar = full + 8 * (c % L::STAGES);
        const int64_t cid = chain * nc + c;
        mbar_expect_tx(bar, L::LOAD);
#pragma unroll
        for (int x = 0; x < DK / 64; ++x) {
            tma_load_4d(t + L::KQ + x * 16384, &tk, 64 * x, c * C, hk, b, bar);
            tma_load_4d(t + L::KQ + x * 16384 + 8192, &tq, 64 * x, c * C, hk, b, bar);
        }
        tma_load_4d(t + L::V, &tv, col0, c * C, h, b, bar);
        tma_load_4d(t + L::V + 8192, &tv, col0 + 64, c * C, h, b, bar);
#pragma unroll
        for (int m = 0; m < 3; ++m) tma_load_2d(t + L::M + m * MAT, &tm, 0, static_cast<int>((cid * 3 + m) * C), bar);
        bulk_load(t + L::G, f.gates + cid * 3 * C, GATES, bar);
    };
    int loaded = 0;                                          // (thread 32) chunks whose copies were started
    if (tid == 32)
        for (; loaded < chunks && loaded < L::STAGES; ++loaded) load(loaded);
    {
        const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane, col = col0 + row;
        const bool live = col < a.dv;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const int64_t per = static_cast<int64_t>(a.dk) * a.dv;
        float* st = r.state + chain * per + col;
        __nv_bfloat16* y = static_cast<__nv_bfloat16*>(r.y) + gdn_base(a.token_major, b, h, a.H, a.T, a.dv) + col;
        const int64_t ys = gdn_stride(a.token_major, a.H, a.dv);
        constexpr int RD = DK / 2, SB = DK / 2;              // rows of d_k per warp; TMEM columns of a part of S
        float S[RD];
        if (chunks > 0) {
#pragma unroll
            for (int x = 0; x < RD; ++x) {
                const int rw = half * RD + x;
                S[x] = live && rw < a.dk ? __ldcs(st + static_cast<int64_t>(rw) * a.dv) : 0.f;
            }
        }
        auto put_state = [&]() {
#pragma unroll
            for (int x = 0; x < RD; x += 32) {
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = S[x + j];
                put_parts(lanes + S_COL + (half * RD + x) / 2, SB, v);
            }
            tmem_st_wait();
        };
        const uint32_t id64 = mma_idesc(64), idk = mma_idesc(DK) | MN_B;
        float out[32];                                       // g Q S of this warp's 32 tokens
        auto finish = [&](int c) {                           // y of chunk c, once step 5 is through
            mbar_wait_or_dead(step + 24, c & 1, dead);
            __syncwarp();
            tc_after_sync();
            float v[32];
            tmem_ld32(lanes + Y_COL + 32 * half, v);
            const int t0 = c * C + 32 * half;
            if (live) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (t0 + j < len) y[(t0 + j) * ys] = __float2bfloat16_rn(a.scale * (out[j] + v[j]));
            }
        };
        if (chunks > 0) put_state();
        for (int c = 0; c < chunks; ++c) {
            const int s = c % L::STAGES;
            const uint32_t t = ring + s * L::BYTES, ph = c & 1;
            const unsigned char* tile = raw + (t - base);
            const float* gate = reinterpret_cast<const float*>(tile + L::G);
            mbar_wait_or_dead(full + 8 * s, (c / L::STAGES) & 1, dead);
            const int n = len - c * C;                       // live tokens (64 or more: all)
            if (n < C) {                                     // K rows past the length: zeros, whatever was there
                for (int p = tid; p < (C - n) * DK / 8; p += 32 * SW) {
                    const int rw = n + p / (DK / 8), x = p % (DK / 8);
                    *reinterpret_cast<uint4*>(raw + (t - base) + (x / 8) * 16384 + rw * 128 + (x % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async();
            }
            tc_before_sync();
            __syncthreads();
            if (tid == 0) {                                  // step 1
                tc_after_sync();
#pragma unroll
                for (int p = 0; p < NS; ++p)
#pragma unroll
                    for (int kk = 0; kk < DK / 16; ++kk)
                        mma_bf16_ta(tmem + X_COL, tmem + S_COL + p * SB + kk * 8, sw128_desc(t + (kk / 4) * 16384 + (kk % 4) * 32), id64, (p | kk) != 0);
                mma_commit(step);
#pragma unroll
                for (int p = 0; p < NS; ++p)
#pragma unroll
                    for (int kk = 0; kk < DK / 16; ++kk)
                        mma_bf16_ta(tmem + X_COL + 64, tmem + S_COL + p * SB + kk * 8, sw128_desc(t + 8192 + (kk / 4) * 16384 + (kk % 4) * 32), id64, (p | kk) != 0);
                mma_commit(step + 32);
            }
            __syncwarp();
            if (c > 0) {
                finish(c - 1);
                if (tid == 32 && loaded < chunks && !*dead) load(loaded++);
                __syncwarp();
            }
            mbar_wait_or_dead(step, ph, dead);
            __syncwarp();
            tc_after_sync();
            {                                                // step 2
                float u[32];
                tmem_ld32(lanes + X_COL + 32 * half, u);
                const unsigned char* vt = tile + L::V + (row / 64) * 8192;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const int i = 32 * half + j;
                    const unsigned short raw16 = *reinterpret_cast<const unsigned short*>(vt + i * 128 + (((row % 64) * 2) ^ ((i & 7) << 4)));
                    const float v = __uint_as_float(static_cast<uint32_t>(raw16) << 16);
                    u[j] = i < n ? gate[C + i] * (v - gate[i] * u[j]) : 0.f;
                }
                put_parts(lanes + R_COL + 16 * half, 32, u);
                tmem_st_wait();
            }
            tc_before_sync();
            __syncthreads();
            if (tid == 0) {                                  // step 3
                tc_after_sync();
#pragma unroll
                for (int m = 0; m < 3; ++m) {                // parts (upper, upper), (upper, lower), (lower, upper)
                    const uint32_t ra = tmem + R_COL + (m == 2 ? 32 : 0), zb = t + L::M + (m == 1 ? MAT : 0);
#pragma unroll
                    for (int kk = 0; kk < C / 16; ++kk)
                        mma_bf16_ta(tmem + X_COL, ra + kk * 8, sw128_desc(zb + kk * 32), id64, (m | kk) != 0);
                }
                mma_commit(step + 8);
            }
            __syncwarp();
            mbar_wait_or_dead(step + 32, ph, dead);
            __syncwarp();
            tc_after_sync();
            tmem_ld32(lanes + X_COL + 64 + 32 * half, out);
#pragma unroll
            for (int j = 0; j < 32; ++j) out[j] *= gate[32 * half + j];
            mbar_wait_or_dead(step + 8, ph, dead);
            __syncwarp();
            tc_after_sync();
            {                                                // step 4
                float w[32], hw[32];
                tmem_ld32(lanes + X_COL + 32 * half, w);
#pragma unroll
                for (int j = 0; j < 32; ++j) hw[j] = w[j] * gate[2 * C + 32 * half + j];
                put_parts(lanes + R_COL + 16 * half, 32, hw);
                put_parts(lanes + W_COL + 16 * half, 32, w);
                tmem_st_wait();
            }
            const float g63 = gate[C - 1];
            tc_before_sync();
            __syncthreads();
            if (tid == 0) {                                  // step 5
                tc_after_sync();
#pragma unroll
                for (int p = 0; p < NS; ++p)
#pragma unroll
                    for (int kk = 0; kk < C / 16; ++kk)
                        mma_bf16_ta(tmem + X_COL, tmem + R_COL + p * 32 + kk * 8, sw128_mn_desc(t + kk * 2048, 16384), idk, (p | kk) != 0);
                mma_commit(step + 16);
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int kk = 0; kk < C / 16; ++kk)
                        mma_bf16_ta(tmem + Y_COL, tmem + W_COL + p * 32 + kk * 8, sw128_desc(t + L::M + 2 * MAT + kk * 32), id64, (p | kk) != 0);
                mma_commit(step + 24);
            }
            __syncwarp();
            mbar_wait_or_dead(step + 16, ph, dead);
            __syncwarp();
            tc_after_sync();
#pragma unroll
            for (int x = 0; x < RD; x += 32) {               // step 6
                float v[32];
                tmem_ld32(lanes + X_COL + half * RD + x, v);
#pragma unroll
                for (int j = 0; j < 32; ++j) S[x + j] = fmaf(g63, S[x + j], v[j]);
            }
            put_state();
        }
        if (chunks > 0) {
            finish(chunks - 1);
            if (live) {
#pragma unroll
                for (int x = 0; x < RD; ++x) {
                    const int rw = half * RD + x;
                    if (rw < a.dk) __stcs(st + static_cast<int64_t>(rw) * a.dv, S[x]);
                }
            }
        }
        if (live)
            for (int t = len + half; t < a.T; t += 2) y[t * ys] = __float2bfloat16_rn(0.f);
    }
    if (tid == 32 && *dead)                                  // the copies in flight land before the CTA ends
        for (int j = loaded > L::STAGES ? loaded - L::STAGES : 0; j < loaded; ++j) mbar_wait(full + 8 * (j % L::STAGES), (j / L::STAGES) & 1);
    tc_before_sync();
    __syncthreads();
    if (tid == 0 && ctl.dead) flag_error(a.err, ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, T_COLS);
}

template <int DK>
cudaError_t factors(const CUtensorMap& tk, const CUtensorMap& tq, const GdnArgs& a, const GdnFactors& f, cudaStream_t stream) {
    constexpr size_t smem = factor_smem<DK>();
    cudaError_t e = cudaFuncSetAttribute(k_gdn_factors<DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    k_gdn_factors<DK><<<dim3((a.T + C - 1) / C, a.H, a.B), FT, smem, stream>>>(tk, tq, a, f);
    return cudaGetLastError();
}

template <int DK>
cudaError_t scan(const CUtensorMap& tk, const CUtensorMap& tq, const CUtensorMap& tv, const CUtensorMap& tm, const GdnScan& s,
                 const GdnFactors& f, cudaStream_t stream) {
    constexpr size_t smem = scan_smem<DK>();
    cudaError_t e = cudaFuncSetAttribute(k_gdn_scan<DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    k_gdn_scan<DK><<<dim3((s.a.dv + 127) / 128, s.a.H, s.a.B), ST, smem, stream>>>(tk, tq, tv, tm, s, f, (s.a.T + C - 1) / C);
    return cudaGetLastError();
}

}  // namespace

size_t gdn_factor_mat_bytes(int64_t chunks) { return static_cast<size_t>(chunks) * 3 * MAT; }
size_t gdn_factor_gate_bytes(int64_t chunks) { return static_cast<size_t>(chunks) * GATES; }

// From one whole chunk up: below, the token recurrence is one launch of about the same length.
bool gdn_chunk_supported(int dtype, int dk, int T) { return dtype == SDM_BF16 && dk <= 128 && T >= C; }

cudaError_t launch_gdn_factors(const GdnArgs& a, const GdnFactors& f, cudaStream_t stream) {
    CUtensorMap tk, tq;
    if (!token_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk) || !token_map(&tq, a.q, a.token_major, a.B, a.Hk, a.T, a.dk))
        return cudaErrorInvalidValue;
    return a.dk <= 64 ? factors<64>(tk, tq, a, f, stream) : factors<128>(tk, tq, a, f, stream);
}

cudaError_t launch_gdn_scan(const GdnScan& s, const GdnFactors& f, cudaStream_t stream) {
    const GdnArgs& a = s.a;
    const int64_t chunks = static_cast<int64_t>(a.B) * a.H * ((a.T + C - 1) / C);
    CUtensorMap tk, tq, tv, tm;
    if (!token_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk) || !token_map(&tq, a.q, a.token_major, a.B, a.Hk, a.T, a.dk) ||
        !token_map(&tv, a.v, a.token_major, a.B, a.H, a.T, a.dv) || !mat_map(&tm, f.mat, chunks * 3))
        return cudaErrorInvalidValue;
    return a.dk <= 64 ? scan<64>(tk, tq, tv, tm, s, f, stream) : scan<128>(tk, tq, tv, tm, s, f, stream);
}

}  // namespace sdm
