// Gated delta rule in chunks of 32 tokens in fp32 (float32 storage, d_k <= 256): the forward walk, the forward
// walk that keeps states and e, and the backward's walk.  Formulas as in the tensor-core kernels: with
// G_ij = prod_{j < l <= i} alpha_l, g_i = prod_{l <= i} alpha_l, h_j = prod_{l > j} alpha_l of a chunk,
//   B_ij = G_ij k_i.k_j (j < i),  P_ij = G_ij q_i.k_j (j <= i),  N = -(I + B beta)^-1 B,
//   forward   r = v - g K S,  e = r + N (beta r),  y = scale (g Q S + P beta e),  S' = g_31 S + K^T (h beta e)
//   reverse   x = h K D + scale P^T dy,  d = x + N^T (beta x),  dv = beta d,
//             D' = g_31 D + scale Q^T (g dy) - K^T (beta g d)
// k_gdn_factors32 makes N and P (or their transposes) and g, beta, h of every chunk at once.  k_gdn_walk
// owns 16 columns of one state, which stay in shared memory, transposed, beside the double-buffered tiles
// of the chunk.  Every product is a dot product along rows of two shared-memory matrices, a thread a 2 x 2 tile
// of them (four 16-byte reads per 16 multiply-adds).  Eight warps: four for K's and N's products, four for Q's and P's
// beside them; four warps with 4 x 2 tiles read less and took 31 us where these took 25.
//
// A chunk is four dependent products in place of 32 dependent tokens: with few sequences and heads the
// latency of the chain is what counts (one head, T = 256, 64 x 64: 26 us here and 8.5 us for the factors, 70 us token by
// token).  With many, the token recurrence's registers win over these shared-memory reads (see gdn_walk_supported).
// Two warps on a scheduler and a barrier after each product: that latency bounds it, not the reads.
#include "gdn_tc.cuh"

namespace sdm {

namespace {

using namespace tc;

constexpr int C = GDN_C32;
constexpr int CW = 16;                   // columns of a CTA
constexpr int NT = 256;                  // computing threads of the walk; a warp beside them fetches
constexpr int FT = 128;                  // threads of the factors
constexpr int CP = C + 4;                // padded row of a [.][32] matrix
constexpr int FACT = 2 * C * C + 3 * C;  // floats of a chunk's factors: N, P, g, beta, h (67 rows of 32)
constexpr int BOX = C * 128;             // bytes of 32 rows x 32 floats, swizzled as TMA leaves them

__device__ __forceinline__ void cp16(void* dst, const void* src, bool on) {
    const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(dst));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(s), "l"(src), "r"(on ? 16 : 0) : "memory");
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
          "l"(reinterpret_cast<unsigned long long&>(c)));
    return d;
}
// acc[r][c] += sum_x A[row r of a][x] B[row c of b, db floats apart][x], x < n (a multiple of 4), in packed pairs:
// with a warp or two on a scheduler it is the number of instructions that counts.  The reads of the next four x are
// issued before this four's products.
template <int R, int S, class A>
__device__ __forceinline__ void tile(A a, const float* b, int db, int n, float (&acc)[R][S]) {
    float4 va[2][R], vb[2][S];
    float2 sum[R][S];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < S; ++c) sum[r][c] = make_float2(acc[r][c], 0.f);
    auto load = [&](int w, int x) {
#pragma unroll
        for (int r = 0; r < R; ++r) va[w][r] = a(r, x);
#pragma unroll
        for (int c = 0; c < S; ++c) vb[w][c] = *reinterpret_cast<const float4*>(b + c * db + x);
    };
    auto mul = [&](int w) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < S; ++c) {
                sum[r][c] = fma2(make_float2(va[w][r].x, va[w][r].y), make_float2(vb[w][c].x, vb[w][c].y), sum[r][c]);
                sum[r][c] = fma2(make_float2(va[w][r].z, va[w][r].w), make_float2(vb[w][c].z, vb[w][c].w), sum[r][c]);
            }
    };
    load(0, 0);
#pragma unroll 1
    for (int x = 0; x < n; x += 8) {
        load(1, x + 4 < n ? x + 4 : x);
        mul(0);
        load(0, x + 8 < n ? x + 8 : x);
        if (x + 4 < n) mul(1);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < S; ++c) acc[r][c] = sum[r][c].x + sum[r][c].y;
}
// Rows of a padded matrix, and of swizzled boxes (32 floats of every row a box): four values of row r from x on.
struct Padded {
    const float* p;
    int ld;
    __device__ __forceinline__ float4 operator()(int r, int x) const { return *reinterpret_cast<const float4*>(p + r * ld + x); }
};
struct Boxed {
    const unsigned char* p;
    int row;
    __device__ __forceinline__ float4 operator()(int r, int x) const {
        const int i = row + r;
        return *reinterpret_cast<const float4*>(p + (x >> 5) * BOX + i * 128 + (((x >> 2 & 7) ^ (i & 7)) << 4));
    }
};

// ------------------------------------------------------------------------------------------
// Factors of a chunk: 128 threads; threads 0-63 take k.k, 64-127 q.k, 4 x 4 each.  N by a column per lane of the
// first warp: N_ic = -(B_ic + sum_{c < k < i} B_ik beta_k N_kc).  From a token on whose k, alpha or beta is not finite, B, P
// and beta are zero and the gate products g are not finite, so that no zero times infinity takes it to the tokens before it.
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(FT) k_gdn_factors32(const GdnArgs a, float* __restrict__ out, int transposed) {
    extern __shared__ __align__(16) float sm[];
    const int ld = a.dk + 4;
    float* const kq = sm;                      // [64][dk + 4]: K, then Q
    float* const B = kq + 64 * ld;             // [32][36] B transposed: [k][i]
    float* const al = B + C * CP;              // alpha, beta
    const int tid = threadIdx.x;
    const int b = blockIdx.z, h = blockIdx.y, ch = blockIdx.x, t0 = ch * C, hk = h / (a.H / a.Hk);
    const int len = gdn_length(a, b);
    if (t0 >= len) return;
    const int n = len - t0 < C ? len - t0 : C;
    const int64_t chain = static_cast<int64_t>(b) * a.H + h;
    const int64_t kb = gdn_base(a.token_major, b, hk, a.Hk, a.T, a.dk), ks = gdn_stride(a.token_major, a.Hk, a.dk);
    for (int row = tid >> 4; row < 2 * C; row += FT / 16) {            // 16 threads a row
        const int t = row % C;
        const float* src = static_cast<const float*>(row < C ? a.k : a.q) + kb + (t0 + t) * ks;
        for (int x = (tid & 15) * 4; x < a.dk; x += 64) cp16(kq + row * ld + x, t < n ? src + x : static_cast<const float*>(a.k), t < n);
    }
    asm volatile("cp.async.commit_group;\n" ::: "memory");
    asm volatile("cp.async.wait_group 0;\n" ::: "memory");
    if (tid < C) {
        al[tid] = tid < n ? __ldg(static_cast<const float*>(a.alpha) + chain * a.T + t0 + tid) : 1.f;
        al[C + tid] = tid < n ? __ldg(static_cast<const float*>(a.beta) + chain * a.T + t0 + tid) : 0.f;
    }
    __syncthreads();
    float* const f = out + (chain * gridDim.x + ch) * FACT;
    __shared__ int first;
    if (tid == 0) first = C;
    bool bad = tid < C && !(gdn_finite(al[tid]) && gdn_finite(al[C + tid]));
    const bool isq = tid >= 64;
    const int i0 = 4 * ((tid & 63) >> 3), j0 = 4 * (tid & 7);          // rows and columns of this thread's tile
    {
        float acc[4][4] = {};
        if (j0 <= i0 + 3) tile<4, 4>(Padded{kq + ((isq ? C : 0) + i0) * ld, ld}, kq + j0 * ld, ld, a.dk, acc);
        float p[4] = {1.f, 1.f, 1.f, 1.f};     // prod_{j0 + 3 < l <= i} alpha_l of the four rows
#pragma unroll 8
        for (int l = i0 + 3; l > j0 + 3; --l) {
            const float f = al[l];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] *= l <= i0 + r ? f : 1.f;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = i0 + r;
            float G[4];                        // prod_{j < l <= i} times the product; 0 above the diagonal
#pragma unroll
            for (int c = 3; c >= 0; --c) {
                const int j = j0 + c;
                G[c] = j <= i ? p[r] * acc[r][c] : 0.f;
                if (j == i && !isq) bad = bad || !gdn_finite(acc[r][c]);      // k.k
                if (j <= i) p[r] *= al[j];
            }
            const float4 v = make_float4(G[0], G[1], G[2], G[3]);
            if (!isq) {
                B[(j0 + 0) * CP + i] = v.x; B[(j0 + 1) * CP + i] = v.y; B[(j0 + 2) * CP + i] = v.z; B[(j0 + 3) * CP + i] = v.w;
            } else if (!transposed) {
                *reinterpret_cast<float4*>(f + C * C + i * C + j0) = v;
            } else {
                float* const to = f + C * C + j0 * C + i;
                to[0] = v.x; to[C] = v.y; to[2 * C] = v.z; to[3 * C] = v.w;
            }
        }
    }
    if (__syncthreads_or(bad)) {
        if (bad && tid < C && !(gdn_finite(al[tid]) && gdn_finite(al[C + tid]))) atomicMin(&first, tid);
        if (tid < C && !gdn_finite(B[tid * CP + tid])) atomicMin(&first, tid);
        __syncthreads();
        if (tid < C && tid >= first) {
            for (int k = 0; k < C; ++k) {
                B[k * CP + tid] = 0.f;
                f[C * C + (transposed ? k * C + tid : tid * C + k)] = 0.f;
            }
            al[C + tid] = 0.f;
            if (tid == first) al[tid] = gdn_nan();
        }
        __syncthreads();
    }
    if (tid < C) {
        const int c = tid;
        float z[C];
#pragma unroll
        for (int j = 0; j < C; ++j) z[j] = 0.f;
#pragma unroll
        for (int k = 0; k < C - 1; ++k) {
            const float y = k == c ? 1.f : al[C + k] * z[k];
#pragma unroll
            for (int q = (k + 1) / 4; q < C / 4; ++q) {
                const float4 l = *reinterpret_cast<const float4*>(B + k * CP + 4 * q);
                if (4 * q > k) z[4 * q] = fmaf(-l.x, y, z[4 * q]);
                if (4 * q + 1 > k) z[4 * q + 1] = fmaf(-l.y, y, z[4 * q + 1]);
                if (4 * q + 2 > k) z[4 * q + 2] = fmaf(-l.z, y, z[4 * q + 2]);
                z[4 * q + 3] = fmaf(-l.w, y, z[4 * q + 3]);
            }
        }
        if (transposed) {
#pragma unroll
            for (int j = 0; j < C; j += 4) *reinterpret_cast<float4*>(f + c * C + j) = make_float4(z[j], z[j + 1], z[j + 2], z[j + 3]);
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j) f[j * C + c] = z[j];
        }
    } else if (tid < 2 * C) {                  // products up to and after a token
        const int t = tid - C;
        float g = 1.f, hh = 1.f;
        for (int l = 0; l < C; ++l) {
            if (l <= t) g *= al[l];
            else hh *= al[l];
        }
        f[2 * C * C + t] = g;
        f[2 * C * C + C + t] = al[C + t];
        f[2 * C * C + 2 * C + t] = hh;
    }
}

// ------------------------------------------------------------------------------------------
// The walk.  MODE 0: forward; 1: forward, keeping the states before the chunks and e; 2: reverse.
// Grid (column blocks of 16, H, B).  Forward, a token whose k, alpha, beta (all columns) or v (its column) is not finite and
// the ones after it are left out of the chunk's products; their outputs and the state after the chunk are NaN.
// ------------------------------------------------------------------------------------------
struct WalkLayout {                            // bytes
    int nb, ld, Q, F, V, G, stage, S, X, U, W, Y, bytes;
    __host__ __device__ explicit WalkLayout(int dk) {
        nb = (dk + 31) / 32;                   // boxes of K (and Q)
        ld = dk + 4;                           // floats of a row of S
        Q = nb * BOX;
        F = 2 * Q;                             // N, P
        V = F + 2 * BOX;                       // v or dy: [32][16]
        G = V + C * CW * 4;                    // g, beta, h
        stage = G + 1024;
        S = 2 * stage;                         // [16][dk + 4]
        X = S + CW * ld * 4;                   // reverse: Q's share of the update, as S
        U = X + CW * ld * 4;                   // [16][36] each: beta r (or beta x); h w (or -beta g d); w (or dy)
        W = U + CW * CP * 4;
        Y = W + CW * CP * 4;
        bytes = 1024 + Y + CW * CP * 4;
    }
};

__device__ __forceinline__ void bar_walk() { asm volatile("bar.sync 1, %0;\n" ::"n"(NT) : "memory"); }
// The same; true if any of the threads brings true.
__device__ __forceinline__ bool bar_walk_or(bool mine) {
    uint32_t any;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(any) : "r"(static_cast<uint32_t>(mine)), "n"(NT) : "memory");
    return any != 0;
}

template <int MODE>
__global__ void __launch_bounds__(NT + 32) k_gdn_walk(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tq,
                                                      const __grid_constant__ CUtensorMap tv, const __grid_constant__ CUtensorMap tf,
                                                      const GdnRecur r, const float* __restrict__ fact) {
    extern __shared__ unsigned char raw[];
    unsigned char* const sm = raw + ((smem_u32(raw) + 1023u & ~1023u) - smem_u32(raw));
    const GdnArgs& a = r.a;
    const WalkLayout L(a.dk);
    const int tid = threadIdx.x, b = blockIdx.z, h = blockIdx.y, hk = h / (a.H / a.Hk), col0 = blockIdx.x * CW;
    const int len = gdn_length(a, b), chunks = (len + C - 1) / C, nc = (a.T + C - 1) / C;
    const int64_t chain = static_cast<int64_t>(b) * a.H + h, per = static_cast<int64_t>(a.dk) * a.dv;
    const int64_t vb = gdn_base(a.token_major, b, h, a.H, a.T, a.dv), vs = gdn_stride(a.token_major, a.H, a.dv);
    float* const y = static_cast<float*>(r.y);
    float* const S = reinterpret_cast<float*>(sm + L.S);
    float* const U = reinterpret_cast<float*>(sm + L.U);
    float* const W = reinterpret_cast<float*>(sm + L.W);
    float* const Y = reinterpret_cast<float*>(sm + L.Y);
    const float* const src = MODE == 0 ? r.state + chain * per : (r.state_in ? r.state_in + chain * per : nullptr);
    for (int i = tid; i < a.dk * (CW / 4); i += NT + 32) {     // 4 columns of a row
        const int x = i / (CW / 4), c = (i % (CW / 4)) * 4;
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (src != nullptr && col0 + c < a.dv) f = *reinterpret_cast<const float4*>(src + static_cast<int64_t>(x) * a.dv + col0 + c);
        S[c * L.ld + x] = f.x; S[(c + 1) * L.ld + x] = f.y; S[(c + 2) * L.ld + x] = f.z; S[(c + 3) * L.ld + x] = f.w;
    }
    auto save = [&](float* dst) {
        for (int i = tid; i < a.dk * (CW / 4); i += NT) {
            const int x = i / (CW / 4), c = (i % (CW / 4)) * 4;
            if (col0 + c < a.dv)
                *reinterpret_cast<float4*>(dst + static_cast<int64_t>(x) * a.dv + col0 + c) =
                    make_float4(S[c * L.ld + x], S[(c + 1) * L.ld + x], S[(c + 2) * L.ld + x], S[(c + 3) * L.ld + x]);
        }
    };
    auto chunk_of = [&](int it) { return MODE == 2 ? chunks - 1 - it : it; };
    // the tiles of the chunks, by a thread beside the computing ones (16-byte cp.async by all of them took 2,460 cycles a
    // chunk to issue, a bulk copy per row 10,000 to go through)
    __shared__ unsigned long long full[2], empty[2];
    __shared__ int dead;
    if (tid == 0) {
        dead = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&full[i]), 1);
            mbar_init(smem_u32(&empty[i]), NT);
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    __syncthreads();
    if (tid >= NT) {
        if (tid == NT) {
            int it = 0;
            for (; it < chunks; ++it) {
                if (it >= 2) mbar_wait_or_dead(smem_u32(&empty[it & 1]), (it / 2 - 1) & 1, &dead);
                if (dead) break;
                const uint32_t to = smem_u32(sm) + (it & 1) * L.stage, bar = smem_u32(&full[it & 1]);
                const int t0 = chunk_of(it) * C;
                const int64_t cid = chain * nc + chunk_of(it);
                mbar_expect_tx(bar, static_cast<uint32_t>((MODE == 1 ? 1 : 2) * L.nb * BOX + 2 * BOX + C * CW * 4 + 3 * C * 4));
                for (int i = 0; i < L.nb; ++i) {
                    tma_load_4d(to + i * BOX, &tk, 32 * i, t0, hk, b, bar);
                    if (MODE != 1) tma_load_4d(to + L.Q + i * BOX, &tq, 32 * i, t0, hk, b, bar);
                }
                tma_load_4d(to + L.F, &tf, 0, static_cast<int>(cid * (FACT / C)), 0, 0, bar);
                tma_load_4d(to + L.F + BOX, &tf, 0, static_cast<int>(cid * (FACT / C)) + C, 0, 0, bar);
                tma_load_4d(to + L.V, &tv, col0, t0, h, b, bar);
                bulk_load(to + L.G, fact + cid * FACT + 2 * C * C, 3 * C * 4, bar);
            }
            if (dead)                                          // the copies in flight land before the CTA ends
                for (int j = it > 2 ? it - 2 : 0; j < it; ++j) mbar_wait(smem_u32(&full[j & 1]), j / 2 & 1);
        }
    } else {
    // 2 x 2 tiles: tokens 2 tr, 2 tr + 1 and columns tc, tc + 8; threads 0-127 take K's (N's) rows, 128-255 Q's (P's)
    const int tr = tid >> 3 & 15, tc = tid & 7, hi = tid >> 7, upto = (2 * tr + 5) & ~3;     // tokens up to the tile's last
    for (int it = 0; it < chunks; ++it) {
        const int ch = chunk_of(it), t0 = ch * C, n = len - t0 < C ? len - t0 : C;
        unsigned char* const st = sm + (it & 1) * L.stage;
        const unsigned char* const K = st;
        const unsigned char* const F = st + L.F;
        float* const V = reinterpret_cast<float*>(st + L.V);
        const float* const g = reinterpret_cast<const float*>(st + L.G);
        const float* const be = g + C;
        const float* const hh = be + C;
        mbar_wait_or_dead(smem_u32(&full[it & 1]), it / 2 & 1, &dead);
        if (n < C) {                                           // rows past the length: zeros, whatever was there
            for (int i = tid; i < (C - n) * 8 * L.nb; i += NT) {
                const int row = n + i / (8 * L.nb), piece = i % (8 * L.nb), at = piece / 8 * BOX + row * 128 + piece % 8 * 16;
                *reinterpret_cast<float4*>(st + at) = make_float4(0.f, 0.f, 0.f, 0.f);
                if (MODE != 1) *reinterpret_cast<float4*>(st + L.Q + at) = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            for (int i = tid; i < (C - n) * CW; i += NT) V[n * CW + i] = 0.f;
        }
        bool odd = false;                                      // a value of v is not finite
        if (MODE != 2)
            for (int i = tid; i < n * CW; i += NT) odd = odd || !gdn_finite(V[i]);
        odd = bar_walk_or(odd);                                // the tiles are in; the last chunk's S is written
        int m2[2] = {n, n};                                    // tokens that the products of this thread's columns take
        if (MODE != 2 && (odd || !gdn_finite(g[C - 1]))) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                int i = 0;
                while (i < n && gdn_finite(g[i]) && gdn_finite(V[i * CW + tc + 8 * c])) ++i;
                m2[c] = i;
            }
        }
        if (MODE != 0) save(r.marks + (chain * nc + ch) * per);
        float acc[2][2] = {}, out[2][2] = {};
        if (MODE == 2) {                                       // dy, and scale P^T dy (the upper half of the threads)
            for (int i = tid; i < C * CW; i += NT) Y[(i % CW) * CP + i / CW] = V[i];
            bar_walk();
            if (hi) tile<2, 2>(Boxed{F + BOX, 2 * tr}, Y + tc * CP, 8 * CP, C, acc);
            else tile<2, 2>(Boxed{K, 2 * tr}, S + tc * L.ld, 8 * L.ld, a.dk, acc);
            if (hi) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) W[(tc + 8 * c) * CP + 2 * tr + m] = a.scale * acc[m][c];
            }
            bar_walk();
            if (!hi) {                                         // x
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 2 * tr + m;
                        acc[m][c] = fmaf(hh[t], acc[m][c], W[(tc + 8 * c) * CP + t]);
                        U[(tc + 8 * c) * CP + t] = be[t] * acc[m][c];
                    }
            }
            bar_walk();
            if (!hi) {                                         // d; N is strictly lower, its transpose upper
                tile<2, 2>(Boxed{F, 2 * tr}, U + tc * CP, 8 * CP, C, acc);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 2 * tr + m, col = col0 + tc + 8 * c;
                        W[(tc + 8 * c) * CP + t] = -be[t] * g[t] * acc[m][c];
                        if (t < n && col < a.dv) {
                            y[vb + (t0 + t) * vs + col] = be[t] * acc[m][c];
                            r.rows[(chain * a.T + t0 + t) * a.dv + col] = acc[m][c];
                        }
                    }
            } else {                                           // scale g dy
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 2 * tr + m;
                        Y[(tc + 8 * c) * CP + t] *= a.scale * g[t];
                    }
            }
            bar_walk();
        } else {
            if (MODE == 0 || !hi) tile<2, 2>(Boxed{hi ? st + L.Q : K, 2 * tr}, S + tc * L.ld, 8 * L.ld, a.dk, acc);   // K S, Q S
            if (!hi) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 2 * tr + m;
                        acc[m][c] = t < m2[c] ? V[t * CW + tc + 8 * c] - g[t] * acc[m][c] : 0.f;
                        U[(tc + 8 * c) * CP + t] = be[t] * acc[m][c];
                    }
            }
            bar_walk();
            if (!hi) {                                         // e
                tile<2, 2>(Boxed{F, 2 * tr}, U + tc * CP, 8 * CP, upto, acc);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 2 * tr + m, col = col0 + tc + 8 * c;
                        const float w = be[t] * acc[m][c];
                        const bool gone = t >= m2[c] && t < n;
                        W[(tc + 8 * c) * CP + t] = gone ? gdn_nan() : hh[t] * w;
                        if (MODE == 0) Y[(tc + 8 * c) * CP + t] = w;
                        if (MODE == 1 && t < n && col < a.dv) r.rows[(chain * a.T + t0 + t) * a.dv + col] = gone ? gdn_nan() : acc[m][c];
                    }
            }
            bar_walk();
            if (MODE == 0 && hi) {
                tile<2, 2>(Boxed{F + BOX, 2 * tr}, Y + tc * CP, 8 * CP, upto, out);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 2 * tr + m, col = col0 + tc + 8 * c;
                        if (t < n && col < a.dv) y[vb + (t0 + t) * vs + col] = t < m2[c] ? a.scale * fmaf(g[t], acc[m][c], out[m][c]) : gdn_nan();
                    }
            }
        }
        // S[c][x] = g_31 S + sum_t (h w)[c][t] K[t][x]: four x and two columns a thread; in reverse the other half of the
        // threads takes Q's share
        const float gl = g[C - 1];
        float* const X = reinterpret_cast<float*>(sm + L.X);
        const int first = MODE == 2 ? tid & 127 : tid, step = MODE == 2 ? 128 : NT;
        auto share = [&](int p, const Boxed& A, const float* B0, float2 (&s0)[2], float2 (&s1)[2]) {
            const int x = (p >> 3) * 4;
            float4 w[2][2], k[2][4];
            auto load = [&](int to, int t) {
                w[to][0] = *reinterpret_cast<const float4*>(B0 + t);
                w[to][1] = *reinterpret_cast<const float4*>(B0 + 8 * CP + t);
#pragma unroll
                for (int e = 0; e < 4; ++e) k[to][e] = A(t + e, x);
            };
            auto add = [&](int of) {
                const float a0[4] = {w[of][0].x, w[of][0].y, w[of][0].z, w[of][0].w}, a1[4] = {w[of][1].x, w[of][1].y, w[of][1].z, w[of][1].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 lo = make_float2(k[of][e].x, k[of][e].y), up = make_float2(k[of][e].z, k[of][e].w);
                    const float2 d0 = make_float2(a0[e], a0[e]), d1 = make_float2(a1[e], a1[e]);
                    s0[0] = fma2(d0, lo, s0[0]); s0[1] = fma2(d0, up, s0[1]);
                    s1[0] = fma2(d1, lo, s1[0]); s1[1] = fma2(d1, up, s1[1]);
                }
            };
            load(0, 0);
#pragma unroll 1
            for (int t = 0; t < C; t += 8) {
                load(1, t + 4);
                add(0);
                load(0, t + 8 < C ? t + 8 : t);
                add(1);
            }
        };
        auto put = [&](float* to, const float2 (&v)[2]) { *reinterpret_cast<float4*>(to) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y); };
        for (int p = first; p < a.dk * 2; p += step) {         // dk / 4 quads x 8 column pairs
            const int x = (p >> 3) * 4, c = p & 7;
            float* const at0 = S + c * L.ld + x;
            float* const at1 = S + (c + 8) * L.ld + x;
            float2 s0[2] = {}, s1[2] = {};
            if (MODE == 2 && hi) {
                share(p, Boxed{st + L.Q, 0}, Y + c * CP, s0, s1);
                put(X + c * L.ld + x, s0);
                put(X + (c + 8) * L.ld + x, s1);
            } else {
                const float4 f0 = *reinterpret_cast<const float4*>(at0), f1 = *reinterpret_cast<const float4*>(at1);
                s0[0] = make_float2(gl * f0.x, gl * f0.y); s0[1] = make_float2(gl * f0.z, gl * f0.w);
                s1[0] = make_float2(gl * f1.x, gl * f1.y); s1[1] = make_float2(gl * f1.z, gl * f1.w);
                share(p, Boxed{K, 0}, W + c * CP, s0, s1);
                put(at0, s0);
                put(at1, s1);
            }
        }
        if (MODE == 2) {
            bar_walk();
            for (int i = tid; i < a.dk * (CW / 4); i += NT) {
                const int at = i / (a.dk / 4) * L.ld + i % (a.dk / 4) * 4;
                float4 f = *reinterpret_cast<const float4*>(S + at);
                const float4 x = *reinterpret_cast<const float4*>(X + at);
                f.x += x.x; f.y += x.y; f.z += x.z; f.w += x.w;
                *reinterpret_cast<float4*>(S + at) = f;
            }
        }
        fence_async();                                     // this chunk's reads before its place is filled again
        mbar_arrive(smem_u32(&empty[it & 1]));
    }
    }
    __syncthreads();
    if (tid == 0 && dead) flag_error(a.err, ERR_TIMEOUT);
    if (MODE == 0 && chunks > 0) save(r.state + chain * per);
    if (MODE == 2 && r.state_out != nullptr) save(r.state_out + chain * per);
    if (MODE != 1)                                             // tokens past the length
        for (int t = len + tid / CW; t < a.T; t += (NT + 32) / CW)
            if (col0 + tid % CW < a.dv) y[vb + t * vs + col0 + tid % CW] = 0.f;
}

// [B, heads, T, d] or [B, T, heads, d] float32 as {d, T, heads, B}, boxes of `cols` values x 32 tokens.
bool float_map(CUtensorMap* m, const void* base, int token_major, int B, int heads, int T, int d, int cols) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = map_encoder();
    if (!enc) return false;
    const cuuint64_t row = static_cast<cuuint64_t>(d) * 4, uT = T, uH = heads;
    cuuint64_t dim[4] = {static_cast<cuuint64_t>(d), uT, uH, static_cast<cuuint64_t>(B)};
    cuuint64_t str[3] = {token_major ? row * uH : row, token_major ? row : row * uT, row * uH * uT};
    cuuint32_t box[4] = {static_cast<cuuint32_t>(cols), C, 1, 1}, es[4] = {1, 1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, const_cast<void*>(base), dim, str, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               cols == 32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE>
cudaError_t walk(const GdnRecur& r, const float* fact, cudaStream_t stream) {
    const GdnArgs& a = r.a;
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_gdn_walk<MODE>, static_cast<size_t>(WalkLayout(256).bytes), seen);
    if (e != cudaSuccess) return e;
    const int64_t rows = static_cast<int64_t>(a.B) * a.H * ((a.T + C - 1) / C) * (FACT / C);
    CUtensorMap tk, tq, tv, tf;
    if (!float_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk, 32) || !float_map(&tq, a.q, a.token_major, a.B, a.Hk, a.T, a.dk, 32) ||
        !float_map(&tv, MODE == 2 ? r.dy : a.v, a.token_major, a.B, a.H, a.T, a.dv, CW) ||
        !float_map(&tf, fact, 0, 1, 1, static_cast<int>(rows), C, 32))
        return cudaErrorInvalidValue;
    k_gdn_walk<MODE><<<dim3((a.dv + CW - 1) / CW, a.H, a.B), NT + 32, WalkLayout(a.dk).bytes, stream>>>(tk, tq, tv, tf, r, fact);
    return cudaGetLastError();
}

}  // namespace

size_t gdn_walk_bytes(int64_t chunks) { return static_cast<size_t>(chunks) * FACT * 4; }

// Up to two CTAs an SM.  Forward, T = 512, H = 16, factors and walk: with 128 x 128 and 256 CTAs 130 us against 191 of the
// token recurrence, at 512 CTAs, measured when the walk took 6% less, 246 against 195; with 64 x 64 94 against 140 at 256 CTAs,
// then 187 against 148 at 576.
bool gdn_walk_supported(int dtype, int B, int H, int T, int dv) {
    return dtype == SDM_F32 && T >= C && static_cast<int64_t>(B) * H * ((dv + CW - 1) / CW) <= 152 * 2;
}

cudaError_t launch_gdn_walk(int mode, const GdnRecur& r, float* fact, cudaStream_t stream) {
    const GdnArgs& a = r.a;
    const size_t smem = static_cast<size_t>(64 * (a.dk + 4) + C * CP + 2 * C) * 4;
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_gdn_factors32, static_cast<size_t>(64 * 260 + C * CP + 2 * C) * 4, seen);
    if (e != cudaSuccess) return e;
    k_gdn_factors32<<<dim3((a.T + C - 1) / C, a.H, a.B), FT, smem, stream>>>(a, fact, mode == 2);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return mode == 0 ? walk<0>(r, fact, stream) : mode == 1 ? walk<1>(r, fact, stream) : walk<2>(r, fact, stream);
}

}  // namespace sdm
