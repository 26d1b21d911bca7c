// Gated delta rule in chunks of 64 tokens on the 5th-generation tensor cores (bf16 storage, d_k <= 128).
//
// With the decay products of a chunk, G_ij = prod_{j < l <= i} alpha_l, g_i = prod_{l <= i} alpha_l and
// h_j = prod_{l > j} alpha_l, and the state S before it,
//   B_ij = G_ij k_i.k_j (j < i),  P_ij = G_ij q_i.k_j (j <= i),  r = v - g K S,
//   e = (I + B beta)^-1 r = r + N (beta r),  N = -(I + B beta)^-1 B,  w = beta e,
//   y = scale (g Q S + P w),   S' = g_63 S + K^T (h w).
// k_gdn_factors computes N, P and the gate products of every chunk at once; k_gdn_scan then walks the
// chunks of one (sequence, head, 128 columns of the state).  The products G are products of gates,
// never quotients or exponentials of sums, and N does not divide by beta, so gates of zero are exact.
//
// Precision: the state and every sum are fp32.  k and q are exact operands.  What the state depends on and is not a bf16
// number enters the MMAs as three bf16 parts (24 significant bits): S, N, beta r and h w; of N (beta r), products below
// 2^-24 are left out.  With two parts of S, N and beta r, keys of a cosine of 0.98 gave the state an error of 8e-6 and the
// backward's, which ends at a hundredth of where it starts, 4.7e-5, where independent keys give 6e-7.  e takes r itself in
// fp32.  y takes S, P and w as two parts: with P as one, keys of a cosine of 0.64 and slow gates gave y an error of
// 9.6e-3, where its own rounding to bf16 is 1.7e-3 (g Q S and P w cancel).
#include "gdn_tc.cuh"

#include <limits.h>

namespace sdm {

namespace {

using namespace tc;
using namespace gdn;

// ------------------------------------------------------------------------------------------
// Factors of a chunk: one CTA of 128 threads.  One MMA chain gives [K; Q] K^T (128 x 64); thread r
// takes row r of it (k_i.k_j for r < 64, q_i.k_j above) and multiplies it by G along the row.
//
// N is solved for by blocks of 16: the diagonal blocks in fp32 by a column per thread in registers, then the
// block diagonals below in order, with Z_ii = (I + B_ii beta)^-1 = I + N_ii beta:
//   N_ij = -Z_ii sum_{j <= k < i} B_ik Y_kj,  Y = I + beta N,  a warp per block, transposed so that the sum is an
// operand of the product with Z as it lies in registers.  These 16 x 16 products are too small for tcgen05 (at least 64
// rows, and a trip through shared memory or TMEM between any two of a chain); they are mma.sync on tf32, each operand as two
// parts of 11 bits, lower times lower left out: 21 bits.  P and N leave through swizzled boxes and TMA.
// At B = 8, H = 16, T = 4096, d_k = 128: 102 us (107 with the backward's six matrices), where q, k, N and P, 0.6 GB, would
// take 89 at the copy rate; with three matrices 88 us, and 119 with the products in fp32 from shared memory and 16-byte stores
// by the threads.  Five CTAs an SM issue half of the time and wait for one another's chains the rest; the parts cut off with a
// mask in place of a conversion gave 10 us, loops kept short for the instruction cache 5.  Halves of 32 in place of block
// diagonals (a shorter chain, more products) took 6 us more; eliminating whole columns of 64 in registers 2016 unrolled
// instructions, whose fetching took 11,600 of a CTA's 20,000 cycles.
// ------------------------------------------------------------------------------------------
constexpr int FT = 128;
constexpr int LP = C + 8;                     // a row; 8 mod 32: the fragments' reads (four rows, eight columns) meet no bank twice
constexpr int BL = 16, NB = C / BL;
struct FactorSmem {
    uint4 al[C / 8];                          // alpha, bf16
    float be[C];
    unsigned long long bar[2];
    uint32_t tmem;
    int dead, first;                          // first: token with a k, alpha or beta that is not finite
};
// The K and Q tiles make room for these once the MMAs have read them, P's boxes for N and Z, and all of it for N's boxes.
struct FactorLate {
    float Bt[C][LP];                          // B transposed
    float N[C][LP];                           // on and below the diagonal blocks
    float Zt[C][BL + 4];                      // Z_ii transposed: [16 block + column][row]
};
constexpr uint32_t P_BOX = sizeof(FactorLate::Bt), FACTOR_LATE = P_BOX + 3 * MAT;
static_assert(P_BOX % 1024 == 0 && sizeof(FactorLate) <= FACTOR_LATE && GDN_N_PARTS * MAT <= FACTOR_LATE, "boxes");
template <int DK>
struct FactorSize {
    static constexpr size_t TILE = 128 * 2 * DK > FACTOR_LATE ? 128 * 2 * DK : FACTOR_LATE;
    static constexpr size_t BYTES = 1024 + TILE + sizeof(FactorSmem);
};

__device__ __forceinline__ uint32_t tf32(float x) { return __float_as_uint(x) & 0xffffe000u; }   // rounded towards zero
// Upper and lower tf32 parts (21 significant bits together) of a fragment.
template <int M>
struct Parts {
    uint32_t hi[M], lo[M];
    __device__ __forceinline__ explicit Parts(const float (&v)[M]) {
#pragma unroll
        for (int i = 0; i < M; ++i) {
            hi[i] = tf32(v[i]);
            lo[i] = tf32(v[i] - __uint_as_float(hi[i]));
        }
    }
};
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// big + small += A B, 16 x 8 x 8, all but the product of the lower parts.
__device__ __forceinline__ void mma_parts(float (&big)[4], float (&small)[4], const Parts<4>& a, const Parts<2>& b) {
    mma_tf32(big, a.hi, b.hi);
    mma_tf32(small, a.lo, b.hi);
    mma_tf32(small, a.hi, b.lo);
}

template <int DK>
__global__ void __launch_bounds__(FT, 5) k_gdn_factors(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tq,
                                                       const __grid_constant__ CUtensorMap tm, const GdnArgs a, const GdnFactors f) {
    extern __shared__ unsigned char raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t tile = (base + 1023u) & ~1023u;        // per 64 values of d_k: 64 rows of K, 64 of Q
    FactorSmem& sm = *reinterpret_cast<FactorSmem*>(raw + (tile - base) + FactorSize<DK>::TILE);
    FactorLate& lt = *reinterpret_cast<FactorLate*>(raw + (tile - base));
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
        sm.first = C;
        mbar_init(bar, 1);
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
        mbar_expect_tx(bar, 128 * 2 * DK);
#pragma unroll
        for (int x = 0; x < DK / 64; ++x) {
            tma_load_4d(tile + x * 16384, &tk, 64 * x, t0, hk, b, bar);
            tma_load_4d(tile + x * 16384 + 8192, &tq, 64 * x, t0, hk, b, bar);
        }
    }
    if (warp == 1) tmem_alloc(smem_u32(&sm.tmem), 64);
    if (tid >= C) {
        const int t = tid - C;
        reinterpret_cast<unsigned short*>(sm.al)[t] = t < n ? __ldg(static_cast<const unsigned short*>(a.alpha) + chain * a.T + t0 + t) : 0x3f80;
        sm.be[t] = t < n ? load_elem<BF16>(a.beta, chain * a.T + t0 + t) : 0.f;
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = sm.tmem;
    if (n < C) {                                          // rows past the length: zeros, whatever was there
        mbar_wait_or_dead(bar, 0, &sm.dead);
        for (int p = tid; p < (C - n) * DK / 4; p += FT) {
            const int half = p % 2, rw = n + (p / 2) / (DK / 8), x = (p / 2) % (DK / 8);
            *reinterpret_cast<uint4*>(raw + (tile - base) + (x / 8) * 16384 + half * 8192 + rw * 128 + (x % 8) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_async();
        __syncthreads();
    }
    if (warp == 0) {
        mbar_wait_or_dead(bar, 0, &sm.dead);
        __syncwarp();
        tc_after_sync();
        const uint32_t idesc = mma_idesc(64);
        const uint64_t d0 = sw128_desc(tile);
        if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < DK / 16; ++kk) {
                const uint64_t at = d0 + (kk / 4) * 1024 + (kk % 4) * 2;
                mma_bf16(tmem, at, at, idesc, kk != 0);
            }
            mma_commit(done);
        }
        __syncwarp();
    } else if (warp == 1) {                               // prefix and suffix products of the gates, two tokens a lane
        const int l = tid & 31;
        const uint32_t w = reinterpret_cast<const uint32_t*>(sm.al)[l];
        const float a0 = __uint_as_float(w << 16), a1 = __uint_as_float(w & 0xffff0000u);
        float p = a0 * a1, q = p;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float u = __shfl_up_sync(0xffffffffu, p, o), v = __shfl_down_sync(0xffffffffu, q, o);
            if (l >= o) p *= u;
            if (l + o < 32) q *= v;
        }
        const float before = __shfl_up_sync(0xffffffffu, p, 1), after = __shfl_down_sync(0xffffffffu, q, 1);
        float* const gates = f.gates + cid * 3 * C;
        const float h1 = l < 31 ? after : 1.f;
        *reinterpret_cast<float2*>(gates + 2 * l) = make_float2(l > 0 ? before * a0 : a0, p);
        *reinterpret_cast<float2*>(gates + C + 2 * l) = make_float2(sm.be[2 * l], sm.be[2 * l + 1]);
        *reinterpret_cast<float2*>(gates + 2 * C + 2 * l) = make_float2(a1 * h1, h1);
    }
    // row i of the decay products, from the diagonal to the left: G_ii = 1, G_i,j-1 = G_ij alpha_j (B's diagonal
    // is not used)
    const int i = tid & 63;
    const bool isk = tid < C;
    mbar_wait_or_dead(done, 0, &sm.dead);
    __syncwarp();
    tc_after_sync();
    float G = 0.f;
    unsigned char* const P = raw + (tile - base) + P_BOX;
#pragma unroll 1
    for (int half = 1; half >= 0; --half) {               // columns 32.. , then 0..; rows 0-31 have none of the first
        if (half == 1 && (warp & 1) == 0) {
            if (!isk) {
#pragma unroll
                for (int j = 4; j < 8; ++j)
                    for (int p = 0; p < f.mats - GDN_N_PARTS; ++p) *reinterpret_cast<uint4*>(P + p * MAT + box_at(i, j)) = make_uint4(0, 0, 0, 0);
            }
            continue;
        }
        float x[32];
        tmem_ld32(tmem + (static_cast<uint32_t>(warp * 32) << 16) + 32 * half, x);
#pragma unroll
        for (int q = 3; q >= 0; --q) {
            const uint4 w = sm.al[4 * half + q];
            const uint32_t al[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 7; e >= 0; --e) {
                const int j = 32 * half + 8 * q + e;
                G = j == i ? 1.f : G;
                x[8 * q + e] *= G;
                G *= __uint_as_float(e & 1 ? al[e / 2] & 0xffff0000u : al[e / 2] << 16);
            }
        }
        if (isk) {
#pragma unroll
            for (int j = 0; j < 32; ++j) lt.Bt[32 * half + j][i] = x[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v[8];
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 32 * half + 8 * j + e <= i ? x[8 * j + e] : 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = split2(v[2 * e], v[2 * e + 1], v[2 * e], v[2 * e + 1]);
                unsigned char* const at = P + box_at(i, 4 * half + j);
                *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = split2(v[2 * e], v[2 * e + 1], v[2 * e], v[2 * e + 1]);
                *reinterpret_cast<uint4*>(at + MAT) = make_uint4(w[0], w[1], w[2], w[3]);
                if (f.mats == GDN_BACK_MATS) *reinterpret_cast<uint4*>(at + 2 * MAT) = pack16<BF16>(v);
            }
        }
    }
    if (!isk) fence_async();
    // A token that is not finite must not reach the ones before it by way of zero times infinity: it and the ones
    // after it are taken out here (the walk makes their outputs and the state NaN).
    const bool bad = tid < n && !(gdn_finite(lt.Bt[tid & 63][tid & 63]) && gdn_finite(sm.be[tid & 63]) &&      // B's diagonal is k.k
                                  (reinterpret_cast<const unsigned short*>(sm.al)[tid & 63] & 0x7f80) != 0x7f80);
    if (__syncthreads_or(bad)) {
        if (bad) atomicMin(&sm.first, tid);
        __syncthreads();
        if (i >= sm.first) {
            if (isk) {
                for (int k = 0; k < C; ++k) lt.Bt[k][i] = 0.f;
                sm.be[i] = 0.f;
                f.gates[cid * 3 * C + i] = gdn_nan();
                f.gates[cid * 3 * C + C + i] = 0.f;
            } else {
                for (int p = 0; p < 8 * (f.mats - GDN_N_PARTS); ++p) *reinterpret_cast<uint4*>(P + p / 8 * MAT + box_at(i, p % 8)) = make_uint4(0, 0, 0, 0);
                fence_async();
            }
        }
        __syncthreads();
    }
    const int row0 = static_cast<int>(cid * f.mats * C);
    if (warp == 2) {                                      // P leaves
        if (elect_one()) {
            for (int p = 0; p < f.mats - GDN_N_PARTS; ++p) tma_store_2d(&tm, tile + P_BOX + p * MAT, 0, row0 + (GDN_N_PARTS + p) * C);
            bulk_commit();
            bulk_wait_read();
        }
        __syncwarp();
        asm volatile("bar.sync 1, 96;\n" ::: "memory");
    }
    if (isk) {                                            // diagonal block tid / 16, column tid % 16
        const int o = tid & ~15, c = tid & 15;
        float z[BL];
#pragma unroll
        for (int j = 0; j < BL; ++j) z[j] = 0.f;
#pragma unroll
        for (int k = 0; k < BL - 1; ++k) {
            const float y = k == c ? 1.f : sm.be[o + k] * z[k];
#pragma unroll
            for (int q = (k + 1) / 4; q < BL / 4; ++q) {
                const float4 l = *reinterpret_cast<const float4*>(&lt.Bt[o + k][o + 4 * q]);
                if (4 * q > k) z[4 * q] = fmaf(-l.x, y, z[4 * q]);
                if (4 * q + 1 > k) z[4 * q + 1] = fmaf(-l.y, y, z[4 * q + 1]);
                if (4 * q + 2 > k) z[4 * q + 2] = fmaf(-l.z, y, z[4 * q + 2]);
                z[4 * q + 3] = fmaf(-l.w, y, z[4 * q + 3]);
            }
        }
        const float be = sm.be[tid];
        asm volatile("bar.sync 1, 96;\n" ::: "memory");   // P has left the place
#pragma unroll
        for (int j = 0; j < BL; ++j) lt.N[o + j][o + c] = z[j];
#pragma unroll
        for (int j = 0; j < BL; j += 4)
            *reinterpret_cast<float4*>(&lt.Zt[tid][j]) = make_float4(j == c ? 1.f : be * z[j], j + 1 == c ? 1.f : be * z[j + 1],
                                                                     j + 2 == c ? 1.f : be * z[j + 2], j + 3 == c ? 1.f : be * z[j + 3]);
    }
    __syncthreads();
    // fragments of 16 x 8 x 8 products, transposed: a lane has column g of N's block (rows t of B, Z, N in turn)
    const int lane = tid & 31, g = lane >> 2, t = lane & 3;
    auto y_part = [&](int k, int c, bool diagonal) {       // Y^T: columns c + g, c + g + 8, rows k + t, k + t + 4 (c: of the diagonal block)
        const float b0 = sm.be[k + t], b1 = sm.be[k + t + 4];
        float v[4] = {b0 * lt.N[k + t][c + g], b0 * lt.N[k + t][c + g + 8], b1 * lt.N[k + t + 4][c + g], b1 * lt.N[k + t + 4][c + g + 8]};
        if (diagonal) {
            v[0] = k + t == c + g ? 1.f : v[0]; v[1] = k + t == c + g + 8 ? 1.f : v[1];
            v[2] = k + t + 4 == c + g ? 1.f : v[2]; v[3] = k + t + 4 == c + g + 8 ? 1.f : v[3];
        }
        return Parts<4>(v);
    };
    auto b_part = [&](int k, int i) {                      // B^T: rows k + t, k + t + 4, column i + g
        const float v[2] = {lt.Bt[k + t][i + g], lt.Bt[k + t + 4][i + g]};
        return Parts<2>(v);
    };
    // An accumulator's columns 2 t, 2 t + 1 take the places of the operand's t, t + 4; the other operand's rows do the same.
    auto x_part = [&](const float (&x)[4], const float (&xs)[4]) {
        const float v[4] = {x[0] + xs[0], x[2] + xs[2], x[1] + xs[1], x[3] + xs[3]};
        return Parts<4>(v);
    };
    auto z_part = [&](int i, int o) {                      // Z_ii^T: rows i + 2 t, i + 2 t + 1, column o + g of the block
        const float v[2] = {lt.Zt[i + 2 * t][o + g], lt.Zt[i + 2 * t + 1][o + g]};
        return Parts<2>(v);
    };
    auto put = [&](int i, int c, const float (&r)[2][4], const float (&rs)[2][4]) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int row = i + 8 * q + 2 * t;
            lt.N[row][c + g] = -(r[q][0] + rs[q][0]); lt.N[row + 1][c + g] = -(r[q][1] + rs[q][1]);
            lt.N[row][c + g + 8] = -(r[q][2] + rs[q][2]); lt.N[row + 1][c + g + 8] = -(r[q][3] + rs[q][3]);
        }
    };
#pragma unroll 1
    for (int d = 1; d < NB; ++d) {                         // blocks (j + d, j)
        if (warp < NB - d) {
            const int j = warp * BL, i = j + d * BL;
            float x[2][4] = {}, xs[2][4] = {}, r[2][4] = {}, rs[2][4] = {};
#pragma unroll
            for (int k8 = 0; k8 < BL; k8 += 8) {
                const Parts<4> A = y_part(j + k8, j, true);
#pragma unroll
                for (int m = 0; m < 2; ++m) mma_parts(x[m], xs[m], A, b_part(j + k8, i + 8 * m));
            }
#pragma unroll 1
            for (int k = j + BL; k < i; k += BL) {
#pragma unroll
                for (int k8 = 0; k8 < BL; k8 += 8) {
                    const Parts<4> A = y_part(k + k8, j, false);
#pragma unroll
                    for (int m = 0; m < 2; ++m) mma_parts(x[m], xs[m], A, b_part(k + k8, i + 8 * m));
                }
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const Parts<4> A = x_part(x[m], xs[m]);
#pragma unroll
                for (int q = 0; q < 2; ++q) mma_parts(r[q], rs[q], A, z_part(i + 8 * m, 8 * q));
            }
            put(i, j, r, rs);
        }
        __syncthreads();
    }
    {   // N in its parts, into boxes where Bt and N were: 16 rows a warp, four values a lane at a time
        const int row = warp * BL + (lane >> 1);
        float v[8][4];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int x = 8 * q + 4 * (lane & 1);
            float4 f4 = make_float4(0.f, 0.f, 0.f, 0.f);
            if (q / 2 <= warp) f4 = *reinterpret_cast<const float4*>(&lt.N[row][x]);      // zeros from the diagonal on
            v[q][0] = x < row ? f4.x : 0.f; v[q][1] = x + 1 < row ? f4.y : 0.f; v[q][2] = x + 2 < row ? f4.z : 0.f; v[q][3] = x + 3 < row ? f4.w : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            unsigned char* const at = raw + (tile - base) + box_at(row, q) + 8 * (lane & 1);
#pragma unroll
            for (int p = 0; p < GDN_N_PARTS; ++p)
                *reinterpret_cast<uint2*>(at + p * MAT) = make_uint2(split2(v[q][0], v[q][1], v[q][0], v[q][1]), split2(v[q][2], v[q][3], v[q][2], v[q][3]));
        }
    }
    fence_async();
    if (tid == 0 && sm.dead) flag_error(a.err, ERR_TIMEOUT);
    tc_before_sync();
    __syncthreads();
    if (tid == 0) {
        for (int p = 0; p < GDN_N_PARTS; ++p) tma_store_2d(&tm, tile + p * MAT, 0, row0 + p * C);
        bulk_commit();
        bulk_wait_read();
    }
    if (warp == 1) tmem_free(tmem, 64);
}

// ------------------------------------------------------------------------------------------
// The walk over the chunks.  A CTA owns 128 columns of one state; everything is transposed, so that a
// TMEM lane is a column: S^T [columns, d_k], w^T [columns, tokens] are A operands written to TMEM from
// registers, and K, Q, N, P are B operands as TMA leaves them in shared memory (K twice: along d_k for
// K S, along the tokens for the update).  Per chunk:
//   1  U = S^T K^T, then S^T Q^T                      (MMA; the second runs under step 2)
//   2  r = v - g U, beta r                            (registers, bf16 parts to TMEM)
//   3  beta r N^T                                     (MMA; g Q S is taken out meanwhile)
//   4  e = r + .., w = beta e, h w                    (registers, bf16 parts to TMEM)
//   5  h w K, then w P^T                              (MMA)
//   6  S = g_63 S + ..                                (registers, bf16 parts to TMEM)
// Warps 0-7 compute: two share a lane quarter; in steps 2 and 4 each takes 32 tokens, in step 6 half of
// d_k.  Warps 8-11 add up the outputs of a chunk beside that, into a box for TMA to store.
// Warp 12 issues the MMAs, warp 13 the copies.
//
// A token with such a value (of k, alpha, beta: all columns, of v: its column) and the ones after it are left out of a chunk's
// products, where zero times infinity would take it to the ones before it; their outputs and the state after the chunk are NaN.
//
// With KEEP (for the backward) nothing is read out: the states before the chunks and e are stored instead, as
// bf16, transposed as the threads hold them, through boxes in shared memory (16-byte stores of the threads' own,
// a row of 256 bytes apart, cost 95 us of 310 at the layer shape), and the state stays as it was.
//
// The chain of six stages is what bounds it: 7,100 cycles a chunk (250 us at B = 8, H = 16, T = 4096, 128 x 128), of which
// the MMAs take 3,200, the hand-overs about 700 and the registers (sums and conversions to bf16 parts) the rest.  With two
// parts of S, N and beta r and one of P it was 200 us (see the precision above); the look for values that are not finite
// and y's own box are 10 of the rest.
// ------------------------------------------------------------------------------------------
constexpr int SW = 8;                          // compute warps
constexpr int OW = 4;                          // output warps
constexpr int ST = 32 * (SW + OW + 4);
constexpr int LAUNCH_REGS = 128, SCAN_REGS = 168, OUT_REGS = 120, IDLE_REGS = 56;   // a thread's registers, at first and after the split
static_assert(SCAN_REGS >= LAUNCH_REGS && OUT_REGS <= LAUNCH_REGS && IDLE_REGS <= LAUNCH_REGS &&
              SW * SCAN_REGS + OW * OUT_REGS + 4 * IDLE_REGS <= (SW + OW + 4) * LAUNCH_REGS, "register split");
constexpr int NS = 2;                          // bf16 parts of S and of w as the factors of Q and P
constexpr int NP = 3;                          // of S as the factor of K, of beta r and of h w
// TMEM columns: X: steps 1, 3, 5; Y: w P^T; S; R: beta r, then w.  h w lies where S is, which steps 2 to 6 do not read.
constexpr uint32_t X_COL = 0, Y_COL = 128, S_COL = 192, R_COL = S_COL + 64 * NP, T_COLS = 512;
static_assert(R_COL + 32 * NP <= T_COLS, "TMEM columns");

template <int DK, bool KEEP>
struct ScanTile {
    static constexpr int MATS = KEEP ? GDN_N_PARTS : GDN_SCAN_MATS;                                       // KEEP: no P, no Q
    static constexpr uint32_t KQ = 0, V = 128 * 2 * DK, M = V + C * 256, G = M + MATS * MAT, BYTES = G + 1024;
    static constexpr uint32_t LOAD = KEEP ? 128 * DK + C * 256 + MATS * MAT + GATES : G + GATES;
    static constexpr int STAGES = 2;
    // boxes on their way to memory: y, per 64 columns; KEEP: of 128 columns, S per 64 of d_k, e per part
    static constexpr uint32_t KS = BYTES * STAGES, KE = KS + 256 * DK, CTL = KEEP ? KE + 32768 : KS + C * 256;
};
// Barriers.  Completed by MMAs or copies: a stage's tile; U; Q S; beta r N; h w K; w P.  Completed by warps:
// operands in TMEM, S and e to be kept in shared memory, Q S taken out, y in shared memory; by the copying
// thread: the kept ones have left it.
enum { B_FULL = 0, B_U = 2, B_QS, B_RN, B_HK, B_WP, B_S, B_R, B_H, B_W, B_KS, B_KE, B_TAKEN, B_Y, B_FREE, B_COUNT };
struct ScanCtl {
    unsigned long long bar[B_COUNT];
    uint32_t tmem;
    int dead;
    int odd[2];                                // of a stage: the last chunk in it with a value of v that is not finite
};
template <int DK, bool KEEP>
constexpr size_t scan_smem() { return 1024 + ScanTile<DK, KEEP>::CTL + sizeof(ScanCtl); }

template <int DK, bool KEEP>
__global__ void __launch_bounds__(ST, 1) k_gdn_scan(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tq,
                                                    const __grid_constant__ CUtensorMap tv, const __grid_constant__ CUtensorMap ty,
                                                    const __grid_constant__ CUtensorMap tm, const GdnScan r, const GdnFactors f, int nc) {
    using L = ScanTile<DK, KEEP>;
    extern __shared__ unsigned char raw[];
    const GdnArgs& a = r.a;
    const uint32_t base = smem_u32(raw);
    const uint32_t ring = (base + 1023u) & ~1023u;
    unsigned char* const ringp = raw + (ring - base);
    ScanCtl& ctl = *reinterpret_cast<ScanCtl*>(ringp + L::CTL);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b = blockIdx.z, h = blockIdx.y, col0 = blockIdx.x * 128, hk = h / (a.H / a.Hk);
    const int len = gdn_length(a, b);
    const int64_t chain = static_cast<int64_t>(b) * a.H + h;
    const int chunks = (len + C - 1) / C;
    const uint32_t bars = smem_u32(&ctl.bar[0]);
    auto bar = [&](int i) { return bars + 8 * i; };
    if (tid == 0) {
        ctl.dead = 0;
        ctl.odd[0] = ctl.odd[1] = -1;
        for (int i = 0; i < B_COUNT; ++i) mbar_init(bar(i), i < B_S || i == B_FREE ? 1 : i == B_TAKEN || i == B_Y ? OW : SW);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
    }
    if (warp == 0) tmem_alloc(smem_u32(&ctl.tmem), T_COLS);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = ctl.tmem;
    volatile int* dead = &ctl.dead;
    constexpr int SB = DK / 2;                               // TMEM columns of a part of S
    // The first of the chunk's tokens from `from` on that is not finite, in a column of v or for all.
    auto first_odd = [&](int c, int from, int n, int column) {
        const unsigned char* const tile = ringp + (c % L::STAGES) * L::BYTES;
        const float* const gate = reinterpret_cast<const float*>(tile + L::G);
        const unsigned char* const v = tile + L::V + (column / 64) * 8192;
        int i = from;
#pragma unroll 1
        while (i < n && gdn_finite(gate[i]) && (*reinterpret_cast<const unsigned short*>(v + sw128_at(i, column % 64)) & 0x7f80) != 0x7f80) ++i;
        return i;
    };

    if (warp >= SW + OW) {
        regs_dec<IDLE_REGS>();
        if (warp == SW + OW) {                               // MMAs
            const uint32_t id64 = mma_idesc(64), idk = mma_idesc(DK) | MN_B;
            for (int c = 0; c < chunks; ++c) {
                const uint32_t t = ring + (c % L::STAGES) * L::BYTES, ph = c & 1;
                const uint64_t dk = sw128_desc(t + L::KQ), dq = sw128_desc(t + L::KQ + 8192), dm = sw128_desc(t + L::M),
                               dkt = sw128_mn_desc(t + L::KQ, 16384);
                await(bar(B_FULL + c % L::STAGES), (c / L::STAGES) & 1, dead);
                await(bar(B_S), ph, dead);
                if (elect_one()) {                           // step 1; lower parts first, here and below: their sums are small
#pragma unroll 1
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < DK / 16; ++kk)
                            mma_bf16_ta(tmem + X_COL, tmem + S_COL + p * SB + kk * 8, dk + (kk / 4) * 1024 + (kk % 4) * 2, id64, p != NP - 1 || kk != 0);
                    mma_commit(bar(B_U));
                    if (!KEEP) {
#pragma unroll 1
                    for (int p = NS - 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < DK / 16; ++kk)
                            mma_bf16_ta(tmem + X_COL + 64, tmem + S_COL + p * SB + kk * 8, dq + (kk / 4) * 1024 + (kk % 4) * 2, id64, p != NS - 1 || kk != 0);
                    mma_commit(bar(B_QS));
                    }
                }
                __syncwarp();
                await(bar(B_R), ph, dead);
                if (elect_one()) {                           // step 3: part ra of beta r with part nb of N
#pragma unroll 1
                    for (int m = 5; m >= 0; --m) {
                        const int ra = m < 5 ? m / 2 : 0, nb = m < 5 ? m % 2 : 2;    // (0, 2), (2, 0), (1, 1), (1, 0), (0, 1), (0, 0)
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + X_COL, tmem + R_COL + ra * 32 + kk * 8, dm + nb * (MAT / 16) + kk * 2, id64, m != 5 || kk != 0);
                    }
                    mma_commit(bar(B_RN));
                }
                __syncwarp();
                if (!KEEP) await(bar(B_TAKEN), ph, dead);
                await(bar(B_H), ph, dead);
                if (elect_one()) {                           // step 5
#pragma unroll 1
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + X_COL, tmem + S_COL + p * 32 + kk * 8, dkt + kk * 128, idk, p != NP - 1 || kk != 0);
                    mma_commit(bar(B_HK));
                }
                __syncwarp();
                if (KEEP) continue;
                await(bar(B_W), ph, dead);
                if (elect_one()) {
#pragma unroll 1
                    for (int m = 2; m >= 0; --m) {           // part m / 2 of w with part m % 2 of P
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + Y_COL, tmem + R_COL + m / 2 * 32 + kk * 8, dm + (GDN_N_PARTS + m % 2) * (MAT / 16) + kk * 2, id64, m != 2 || kk != 0);
                    }
                    mma_commit(bar(B_WP));
                }
                __syncwarp();
            }
        } else if (warp == SW + OW + 1 && lane == 0) {       // copies
            auto load = [&](int c) {
                const uint32_t t = ring + (c % L::STAGES) * L::BYTES, fb = bar(B_FULL + c % L::STAGES);
                const int64_t cid = chain * nc + c;
                mbar_expect_tx(fb, L::LOAD);
#pragma unroll
                for (int x = 0; x < DK / 64; ++x) {
                    tma_load_4d(t + L::KQ + x * 16384, &tk, 64 * x, c * C, hk, b, fb);
                    if (!KEEP) tma_load_4d(t + L::KQ + x * 16384 + 8192, &tq, 64 * x, c * C, hk, b, fb);
                }
                tma_load_4d(t + L::V, &tv, col0, c * C, h, b, fb);
                tma_load_4d(t + L::V + 8192, &tv, col0 + 64, c * C, h, b, fb);
#pragma unroll
                for (int m = 0; m < L::MATS; ++m) tma_load_2d(t + L::M + m * MAT, &tm, 0, static_cast<int>((cid * f.mats + m) * C), fb);
                bulk_load(t + L::G, f.gates + cid * 3 * C, GATES, fb);
            };
            int loaded = 0;
            for (; loaded < chunks && loaded < L::STAGES; ++loaded) load(loaded);
            for (int c = 0; c < chunks; ++c) {
                if (KEEP) {                                  // S and e on their way, then the next tile
                    const int64_t cid = chain * nc + c;
                    const int nblk = gridDim.x, blk = blockIdx.x;
                    const int rs = static_cast<int>((cid * nblk + blk) * 128), rp = static_cast<int>((cid * 2 * nblk + blk) * 128);
                    mbar_wait_or_dead(bar(B_KS), c & 1, dead);
                    if (*dead) break;
#pragma unroll
                    for (int x = 0; x < DK / 64; ++x) tma_store_2d(&tq, ring + L::KS + x * 16384, 64 * x, rs);
                    mbar_wait_or_dead(bar(B_KE), c & 1, dead);
                    if (*dead) break;
#pragma unroll
                    for (int p = 0; p < 2; ++p) tma_store_2d(&ty, ring + L::KE + p * 16384, 0, rp + p * nblk * 128);
                    bulk_commit();
                    bulk_wait_read();
                    mbar_arrive(bar(B_FREE));
                    mbar_wait_or_dead(bar(B_HK), c & 1, dead);
                    if (*dead) break;
                    if (loaded < chunks) load(loaded++);
                    continue;
                }
                mbar_wait_or_dead(bar(B_WP), c & 1, dead);   // the last that reads chunk c's tile
                if (*dead) break;
                if (loaded < chunks) load(loaded++);
                mbar_wait_or_dead(bar(B_Y), c & 1, dead);
                if (*dead) break;
                tma_store_4d(&ty, ring + L::KS, col0, c * C, h, b);
                if (col0 + 64 < a.dv) tma_store_4d(&ty, ring + L::KS + 8192, col0 + 64, c * C, h, b);
                bulk_commit();
                bulk_wait_read();
                mbar_arrive(bar(B_FREE));
            }
            bulk_wait();
            if (*dead)                                       // the copies in flight land before the CTA ends
                for (int j = loaded > L::STAGES ? loaded - L::STAGES : 0; j < loaded; ++j)
                    mbar_wait(bar(B_FULL + j % L::STAGES), (j / L::STAGES) & 1);
        }
    } else if (warp >= SW) {                                 // outputs: column `row`, all tokens
        regs_dec<OUT_REGS>();
        const int quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        for (int c = 0; !KEEP && c < chunks; ++c) {
            const uint32_t ph = c & 1;
            const float* gate = reinterpret_cast<const float*>(ringp + (c % L::STAGES) * L::BYTES + L::G);
            unsigned char* const yt = ringp + L::KS + (row / 64) * 8192;
            const int n = len - c * C < C ? len - c * C : C;
            mbar_wait_or_dead(bar(B_FULL + c % L::STAGES), (c / L::STAGES) & 1, dead);
            await(bar(B_QS), ph, dead);
            float out[C];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v[32];
                tmem_ld32(lanes + X_COL + 64 + 32 * e, v);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 g = *reinterpret_cast<const float4*>(gate + 32 * e + j);
                    out[32 * e + j] = g.x * v[j]; out[32 * e + j + 1] = g.y * v[j + 1];
                    out[32 * e + j + 2] = g.z * v[j + 2]; out[32 * e + j + 3] = g.w * v[j + 3];
                }
            }
            mbar_wait_or_dead(bar(B_R), ph, dead);           // the computing warps have seen the chunk's v
            const bool odd = __any_sync(0xffffffffu, ctl.odd[c % L::STAGES] == c || !gdn_finite(gate[C - 1]));
            const int m = odd ? first_odd(c, 0, n, row) : n;
            announce(bar(B_TAKEN), lane);                    // and nothing of the tile is read from here on
            if (odd || n < C) {
#pragma unroll
                for (int j = 0; j < C; ++j) out[j] = j < m ? out[j] : j < n ? gdn_nan() : 0.f;
            }
            if (c > 0) mbar_wait_or_dead(bar(B_FREE), (c - 1) & 1, dead);
            await(bar(B_WP), ph, dead);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v[32];
                tmem_ld32(lanes + Y_COL + 32 * e, v);
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    *reinterpret_cast<__nv_bfloat16*>(yt + sw128_at(32 * e + j, row % 64)) = __float2bfloat16_rn(a.scale * (out[32 * e + j] + v[j]));
            }
            fence_async();
            announce(bar(B_Y), lane);
        }
        const int col = col0 + row;                          // chunks past the length
        if (!KEEP && col < a.dv) {
            __nv_bfloat16* y = static_cast<__nv_bfloat16*>(r.y) + gdn_base(a.token_major, b, h, a.H, a.T, a.dv) + col;
            const int64_t ys = gdn_stride(a.token_major, a.H, a.dv);
            for (int t = chunks * C; t < a.T; ++t) y[t * ys] = __float2bfloat16_rn(0.f);
        }
    } else {
        regs_inc<SCAN_REGS>();
        const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane, col = col0 + row;
        const int i0 = 32 * half;                            // this warp's tokens of a chunk
        const bool live = col < a.dv;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const int64_t per = static_cast<int64_t>(a.dk) * a.dv;
        float* st = const_cast<float*>(KEEP ? r.state_in : r.state) + chain * per + col;
        constexpr int RD = DK / 2;                           // rows of d_k of a warp
        float S[RD];
        if (chunks > 0) {
#pragma unroll
            for (int x = 0; x < RD; ++x) {
                const int rw = half * RD + x;
                S[x] = live && rw < a.dk ? __ldcs(st + static_cast<int64_t>(rw) * a.dv) : 0.f;
            }
        }
        auto put_state = [&](int next) {                     // S before chunk `next`
            if (KEEP && next > 0) mbar_wait_or_dead(bar(B_FREE), (next - 1) & 1, dead);
            __syncwarp();
#pragma unroll
            for (int x = 0; x < RD; x += 32) {
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = S[x + j];
                auto keep = [&](int j, const uint4& w) {     // 8 rows of d_k
                    const int at = half * RD + x + 8 * j;
                    if (KEEP) *reinterpret_cast<uint4*>(ringp + L::KS + at / 64 * 16384 + box_at(row, at % 64 / 8)) = w;
                };
                put_part(lanes + S_COL + (half * RD + x) / 2, v, keep);
                put_part(lanes + S_COL + SB + (half * RD + x) / 2, v);
                put_last(lanes + S_COL + (NP - 1) * SB + (half * RD + x) / 2, v);
            }
            if (len - next * C < C) {                        // K rows past the length: zeros, whatever was there
                const int n = len - next * C, s = next % L::STAGES;
                mbar_wait_or_dead(bar(B_FULL + s), (next / L::STAGES) & 1, dead);
                for (int p = tid; p < (C - n) * DK / 8; p += 32 * SW) {
                    const int rw = n + p / (DK / 8), x = p % (DK / 8);
                    *reinterpret_cast<uint4*>(ringp + s * L::BYTES + L::KQ + (x / 8) * 16384 + rw * 128 + (x % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async();
                __syncwarp();
            }
            announce(bar(B_S), lane);
            if (KEEP) hand_over(bar(B_KS), lane);
        };
        const uint32_t vat = L::V + (row / 64) * 8192;
        if (chunks > 0) put_state(0);
        for (int c = 0; c < chunks; ++c) {
            const int s = c % L::STAGES;
            const uint32_t ph = c & 1;
            const unsigned char* tile = ringp + s * L::BYTES;
            const float* gate = reinterpret_cast<const float*>(tile + L::G);
            mbar_wait_or_dead(bar(B_FULL + s), (c / L::STAGES) & 1, dead);
            const int n = len - c * C < C ? len - c * C : C;
            float u[32], w[32];                              // r; then w (with KEEP: e)
            uint32_t v[16];                                  // this column's v, two tokens in a word
#pragma unroll
            for (int j = 0; j < 16; ++j)
                v[j] = *reinterpret_cast<const unsigned short*>(tile + vat + sw128_at(i0 + 2 * j, row % 64)) |
                       (static_cast<uint32_t>(*reinterpret_cast<const unsigned short*>(tile + vat + sw128_at(i0 + 2 * j + 1, row % 64))) << 16);
            uint32_t odd_v = 0;                              // an exponent of all ones
#pragma unroll
            for (int j = 0; j < 16; ++j) odd_v |= __vcmpeq2(v[j] & 0x7f807f80u, 0x7f807f80u);
            const float g63 = gate[C - 1];
            const bool odd = __any_sync(0xffffffffu, odd_v != 0 || !gdn_finite(g63));
            int m = n;                                       // tokens that the products take (of this warp's)
            if (odd) {
                m = first_odd(c, i0, n, row);
                if (m < n && m < i0 + 32) ctl.odd[s] = c;
            }
            await(bar(B_U), ph, dead);
            tmem_ld32(lanes + X_COL + i0, u);                // step 2
            float be[32];
            get32(gate + C + i0, be);
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 g = *reinterpret_cast<const float4*>(gate + i0 + j);
                u[j] = __uint_as_float(v[j / 2] << 16) - g.x * u[j];
                u[j + 1] = __uint_as_float(v[j / 2] & 0xffff0000u) - g.y * u[j + 1];
                u[j + 2] = __uint_as_float(v[j / 2 + 1] << 16) - g.z * u[j + 2];
                u[j + 3] = __uint_as_float(v[j / 2 + 1] & 0xffff0000u) - g.w * u[j + 3];
            }
            if (odd || n < C) {
#pragma unroll
                for (int j = 0; j < 32; ++j) u[j] = i0 + j < m ? u[j] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) w[j] = be[j] * u[j];
            put_part(lanes + R_COL + i0 / 2, w);
            put_part(lanes + R_COL + 32 + i0 / 2, w);
            put_last(lanes + R_COL + 32 * (NP - 1) + i0 / 2, w);
            announce(bar(B_R), lane);
            if (!KEEP) await(bar(B_QS), ph, dead);           // S is read: h w may lie there
            await(bar(B_RN), ph, dead);
            tmem_ld32(lanes + X_COL + i0, w);                // step 4
            if (KEEP) {
#pragma unroll
                for (int j = 0; j < 32; ++j) w[j] += u[j];
            }
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 b4 = *reinterpret_cast<const float4*>(gate + C + i0 + j), h4 = *reinterpret_cast<const float4*>(gate + 2 * C + i0 + j);
                const float bj[4] = {b4.x, b4.y, b4.z, b4.w}, hj[4] = {h4.x, h4.y, h4.z, h4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (KEEP) {                              // e stays in w
                        u[j + e] = hj[e] * (bj[e] * w[j + e]);
                    } else {
                        w[j + e] = bj[e] * (w[j + e] + u[j + e]);
                        u[j + e] = hj[e] * w[j + e];
                    }
                }
            }
            if (odd && m < n) {
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    if (i0 + j >= m) u[j] = gdn_nan();
                    if (KEEP && i0 + j >= m && i0 + j < n) w[j] = gdn_nan();
                }
            }
            put_part(lanes + S_COL + i0 / 2, u);
            put_part(lanes + S_COL + 32 + i0 / 2, u);
            put_last(lanes + S_COL + 64 + i0 / 2, u);
            announce(bar(B_H), lane);
            if (KEEP) {
                keep_parts(ringp + L::KE, row, i0 / 8, w);
                hand_over(bar(B_KE), lane);
            } else {
                put_part(lanes + R_COL + i0 / 2, w);
                put_last(lanes + R_COL + 32 + i0 / 2, w);
                announce(bar(B_W), lane);
            }
            await(bar(B_HK), ph, dead);
#pragma unroll
            for (int x = 0; x < RD; x += 32) {               // step 6
                float d[32];
                tmem_ld32(lanes + X_COL + half * RD + x, d);
#pragma unroll
                for (int j = 0; j < 32; ++j) S[x + j] = fmaf(g63, S[x + j], d[j]);
            }
            if (c + 1 < chunks) put_state(c + 1);
        }
        if (!KEEP && chunks > 0 && live) {
#pragma unroll
            for (int x = 0; x < RD; ++x) {
                const int rw = half * RD + x;
                if (rw < a.dk) __stcs(st + static_cast<int64_t>(rw) * a.dv, S[x]);
            }
        }
    }
    tc_before_sync();
    __syncthreads();
    if (tid == 0 && ctl.dead) flag_error(a.err, ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, T_COLS);
}

template <int DK>
cudaError_t factors(const CUtensorMap& tk, const CUtensorMap& tq, const CUtensorMap& tm, const GdnArgs& a, const GdnFactors& f, cudaStream_t stream) {
    constexpr size_t smem = FactorSize<DK>::BYTES;
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_gdn_factors<DK>, smem, seen);
    if (e != cudaSuccess) return e;
    k_gdn_factors<DK><<<dim3((a.T + C - 1) / C, a.H, a.B), FT, smem, stream>>>(tk, tq, tm, a, f);
    return cudaGetLastError();
}

template <int DK, bool KEEP>
cudaError_t scan(const CUtensorMap& tk, const CUtensorMap& tq, const CUtensorMap& tv, const CUtensorMap& ty, const CUtensorMap& tm, const GdnScan& s,
                 const GdnFactors& f, cudaStream_t stream) {
    constexpr size_t smem = scan_smem<DK, KEEP>();
    static std::atomic<int> regs{0};
    cudaError_t e = check_kernel_registers(k_gdn_scan<DK, KEEP>, LAUNCH_REGS, regs);
    if (e != cudaSuccess) return e;
    static std::atomic<unsigned long long> seen;
    e = allow_smem(k_gdn_scan<DK, KEEP>, smem, seen);
    if (e != cudaSuccess) return e;
    k_gdn_scan<DK, KEEP><<<dim3((s.a.dv + 127) / 128, s.a.H, s.a.B), ST, smem, stream>>>(tk, tq, tv, ty, tm, s, f, (s.a.T + C - 1) / C);
    return cudaGetLastError();
}

}  // namespace

size_t gdn_factor_mat_bytes(int64_t chunks, int mats) { return static_cast<size_t>(chunks) * mats * MAT; }
size_t gdn_factor_gate_bytes(int64_t chunks) { return static_cast<size_t>(chunks) * GATES; }

// A chunk costs the same however few tokens it holds.  Forward, H = 16, 128 x 128, 32 (63) tokens: 18.8 (18.7) us against
// 18.7 (30.9) token by token at B = 2, 31 (31) against 39 (70) at B = 16, 93 (99) against 123 (226) at B = 64; backward: 48 (48)
// against 78 (102) at B = 2, 88 against 184 at B = 16.  Small heads in large batches would do better token by token: 66 (66)
// against 19 (33) at B = 64 with 32 x 32.
bool gdn_chunk_supported(int dtype, int dk, int T) { return dtype == SDM_BF16 && dk <= 128 && T >= 32; }

cudaError_t launch_gdn_factors(const GdnArgs& a, const GdnFactors& f, cudaStream_t stream) {
    const int64_t chunks = static_cast<int64_t>(a.B) * a.H * ((a.T + C - 1) / C);
    if (chunks * f.mats * C > INT_MAX) return cudaErrorInvalidValue;       // rows of the matrices, 275 GB of them
    CUtensorMap tk, tq, tm;
    if (!token_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk) || !token_map(&tq, a.q, a.token_major, a.B, a.Hk, a.T, a.dk) ||
        !row_map(&tm, f.mat, chunks * f.mats * C, C, C))
        return cudaErrorInvalidValue;
    return a.dk <= 64 ? factors<64>(tk, tq, tm, a, f, stream) : factors<128>(tk, tq, tm, a, f, stream);
}

cudaError_t launch_gdn_scan(const GdnScan& s, const GdnFactors& f, cudaStream_t stream) {
    const GdnArgs& a = s.a;
    const int64_t chunks = static_cast<int64_t>(a.B) * a.H * ((a.T + C - 1) / C);
    CUtensorMap tk, tq, tv, ty, tm;
    if (s.keep_S != nullptr) {                  // the boxes go where q and y are otherwise
        const int nblk = (a.dv + 127) / 128, dkp = a.dk <= 64 ? 64 : 128;
        if (!token_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk) || !row_map(&tq, s.keep_S, chunks * nblk * 128, dkp, 128) ||
            !token_map(&tv, a.v, a.token_major, a.B, a.H, a.T, a.dv) || !row_map(&ty, s.keep_e, chunks * 2 * nblk * 128, C, 128) ||
            !row_map(&tm, f.mat, chunks * f.mats * C, C, C))
            return cudaErrorInvalidValue;
        return a.dk <= 64 ? scan<64, true>(tk, tq, tv, ty, tm, s, f, stream) : scan<128, true>(tk, tq, tv, ty, tm, s, f, stream);
    }
    if (!token_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk) || !token_map(&tq, a.q, a.token_major, a.B, a.Hk, a.T, a.dk) ||
        !token_map(&tv, a.v, a.token_major, a.B, a.H, a.T, a.dv) || !token_map(&ty, s.y, a.token_major, a.B, a.H, a.T, a.dv) || !row_map(&tm, f.mat, chunks * f.mats * C, C, C))
        return cudaErrorInvalidValue;
    return a.dk <= 64 ? scan<64, false>(tk, tq, tv, ty, tm, s, f, stream) : scan<128, false>(tk, tq, tv, ty, tm, s, f, stream);
}

}  // namespace sdm
