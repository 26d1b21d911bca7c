// Gated delta rule in chunks of 32 tokens in fp32 (float32 storage, d_k <= 256): the forward walk, the forward
// walk that keeps states and e, and the backward's walk.  Formulas as in the tensor-core kernels: with
// G_ij = prod_{j < l <= i} alpha_l, g_i = prod_{l <= i} alpha_l, h_j = prod_{l > j} alpha_l of a chunk,
//   B_ij = G_ij k_i.k_j (j < i),  P_ij = G_ij q_i.k_j (j <= i),  N = -(I + B beta)^-1 B,
//   forward   r = v - g K S,  e = r + N (beta r),  y = scale (g Q S + P beta e),  S' = g_31 S + K^T (h beta e)
//   reverse   x = h K D + scale P^T dy,  d = x + N^T (beta x),  dv = beta d,
//             D' = g_31 D + scale Q^T (g dy) - K^T (beta g d)
// k_gdn_factors32 makes N and P (or their transposes) and g, beta, h of every chunk at once.  k_gdn_walk
// owns 16 columns of one state, which stay in shared memory, transposed, beside the double-buffered tiles
// of the chunk.  Every product is a dot product along rows of two padded shared-memory matrices, a thread a
// 4 x 2 tile of them (six 16-byte reads per 32 multiply-adds).
//
// A chunk is four dependent products in place of 32 dependent tokens: with few sequences and heads the
// latency of the chain is what counts, and this form has about a fifth of the token recurrence's.  With many, the
// token recurrence's registers win over these shared-memory reads (see launch_gdn_walk's rule).
#include "gdn_internal.h"

namespace sdm {

namespace {

constexpr int C = GDN_C32;
constexpr int CW = 16;                   // columns of a CTA
constexpr int NT = 128;
constexpr int CP = C + 4;                // padded row of a [.][32] matrix
constexpr int FACT = 2 * C * C + 3 * C;  // floats of a chunk's factors: N, P, g, beta, h

__device__ __forceinline__ void cp16(void* dst, const void* src, bool on) {
    const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(dst));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(s), "l"(src), "r"(on ? 16 : 0) : "memory");
}

__device__ __forceinline__ float dot4(const float4& x, const float4& y, float s) {
    return fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s))));
}
// acc[r][c] += sum_x A[4 rows of a][x] B[rows b and b + db][x], x < n (a multiple of 4).
template <int R>
__device__ __forceinline__ void tile(const float* a, int lda, const float* b, int db, int n, float (&acc)[R][2]) {
#pragma unroll 4
    for (int x = 0; x < n; x += 4) {
        const float4 b0 = *reinterpret_cast<const float4*>(b + x), b1 = *reinterpret_cast<const float4*>(b + db + x);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float4 v = *reinterpret_cast<const float4*>(a + r * lda + x);
            acc[r][0] = dot4(v, b0, acc[r][0]);
            acc[r][1] = dot4(v, b1, acc[r][1]);
        }
    }
}

// ------------------------------------------------------------------------------------------
// Factors of a chunk: 128 threads; threads 0-63 take k.k, 64-127 q.k, 4 x 4 each.  N by a column per lane of the
// first warp: N_ic = -(B_ic + sum_{c < k < i} B_ik beta_k N_kc).
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(NT) k_gdn_factors32(const GdnArgs a, float* __restrict__ out, int transposed) {
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
    for (int row = tid >> 4; row < 2 * C; row += NT / 16) {            // 16 threads a row
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
    const bool isq = tid >= 64;
    const int i0 = 4 * ((tid & 63) >> 3), j0 = 4 * (tid & 7);          // rows and columns of this thread's tile
    {
        float acc[2][4][2] = {};
        if (j0 <= i0 + 3) {
            const float* A = kq + ((isq ? C : 0) + i0) * ld;
            tile<4>(A, ld, kq + j0 * ld, ld, a.dk, acc[0]);
            tile<4>(A, ld, kq + (j0 + 2) * ld, ld, a.dk, acc[1]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = i0 + r;
            float G[4];                        // prod_{j < l <= i}, 0 above the diagonal
            float p = 1.f;
            for (int l = i; l > j0 + 3; --l) p *= al[l];
#pragma unroll
            for (int c = 3; c >= 0; --c) {
                const int j = j0 + c;
                G[c] = j <= i ? p : 0.f;
                if (j <= i) p *= al[j];
            }
            float4 v;
            v.x = G[0] * acc[0][r][0]; v.y = G[1] * acc[0][r][1]; v.z = G[2] * acc[1][r][0]; v.w = G[3] * acc[1][r][1];
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
    __syncthreads();
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
// Grid (column blocks of 16, H, B).
// ------------------------------------------------------------------------------------------
struct WalkLayout {
    int ld, kq, v, f, stage, S, u, w, y, floats;
    __host__ __device__ explicit WalkLayout(int dk) {
        ld = dk + 4;
        kq = 0;                                // K, Q: [64][dk + 4]
        v = kq + 64 * ld;                      // v or dy: [32][16]
        f = v + C * CW;                        // N, P: [64][36]; g, beta, h
        stage = f + 2 * C * CP + 3 * C;
        S = 2 * stage;                         // [16][dk + 4]
        u = S + CW * ld;                       // [16][36] each: beta r (or beta x); h w (or -beta g d); w (or dy)
        w = u + CW * CP;
        y = w + CW * CP;
        floats = y + CW * CP;
    }
};

template <int MODE>
__global__ void __launch_bounds__(NT) k_gdn_walk(const GdnRecur r, const float* __restrict__ fact) {
    extern __shared__ __align__(16) float sm[];
    const GdnArgs& a = r.a;
    const WalkLayout L(a.dk);
    const int tid = threadIdx.x, b = blockIdx.z, h = blockIdx.y, hk = h / (a.H / a.Hk), col0 = blockIdx.x * CW;
    const int len = gdn_length(a, b), chunks = (len + C - 1) / C, nc = (a.T + C - 1) / C;
    const int64_t chain = static_cast<int64_t>(b) * a.H + h, per = static_cast<int64_t>(a.dk) * a.dv;
    const int64_t vb = gdn_base(a.token_major, b, h, a.H, a.T, a.dv), vs = gdn_stride(a.token_major, a.H, a.dv);
    const int64_t kb = gdn_base(a.token_major, b, hk, a.Hk, a.T, a.dk), ks = gdn_stride(a.token_major, a.Hk, a.dk);
    float* const y = static_cast<float*>(r.y);
    float* const S = sm + L.S;
    float* const U = sm + L.u;
    float* const W = sm + L.w;
    float* const Y = sm + L.y;
    const float* const src = MODE == 0 ? r.state + chain * per : (r.state_in ? r.state_in + chain * per : nullptr);
    for (int i = tid; i < a.dk * (CW / 4); i += NT) {          // 4 columns of a row
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
    auto stage = [&](int it) {
        float* const to = sm + (it & 1) * L.stage;
        const int ch = chunk_of(it), t0 = ch * C;
        for (int row = tid >> 4; row < (MODE == 1 ? C : 2 * C); row += NT / 16) {      // 16 threads a row
            const int t = t0 + row % C;
            const bool on = t < len;
            const float* p = static_cast<const float*>(row < C ? a.k : a.q) + kb + (on ? t * ks : 0);
            for (int x = (tid & 15) * 4; x < a.dk; x += 64) cp16(to + L.kq + row * L.ld + x, p + x, on);
        }
        const float* vp = static_cast<const float*>(MODE == 2 ? r.dy : a.v) + vb;
        for (int i = tid; i < C * (CW / 4); i += NT) {
            const int t = i / (CW / 4), c = (i % (CW / 4)) * 4;
            const bool on = t0 + t < len && col0 + c < a.dv;
            cp16(to + L.v + t * CW + c, vp + (on ? (t0 + t) * vs + col0 + c : 0), on);
        }
        const float* f = fact + (chain * nc + ch) * FACT;
        for (int i = tid; i < (2 * C * C + 3 * C) / 4; i += NT) {
            const int row = i / (C / 4), x = (i % (C / 4)) * 4;
            cp16(row < 2 * C ? to + L.f + row * CP + x : to + L.f + 2 * C * CP + (row - 2 * C) * C + x, f + 4 * i, true);
        }
        asm volatile("cp.async.commit_group;\n" ::: "memory");
    };
    if (chunks > 0) stage(0);
    // 4 x 2 tiles: tokens 4 tr .. and columns tc, tc + 8; threads 0-63 take K's (N's) rows, 64-127 Q's (P's)
    const int tr = tid >> 3 & 7, tc = tid & 7, hi = tid >> 6;
    for (int it = 0; it < chunks; ++it) {
        const int ch = chunk_of(it), t0 = ch * C, n = len - t0 < C ? len - t0 : C;
        const float* const st = sm + (it & 1) * L.stage;
        const float* const K = st + L.kq;
        const float* const V = st + L.v;
        const float* const F = st + L.f;
        const float* const g = F + 2 * C * CP;
        const float* const be = g + C;
        const float* const hh = be + C;
        asm volatile("cp.async.wait_group 0;\n" ::: "memory");
        __syncthreads();                                       // the tiles are in; the last chunk is done with
        if (it + 1 < chunks) stage(it + 1);
        if (MODE != 0) save(r.marks + (chain * nc + ch) * per);
        float acc[4][2] = {}, out[4][2] = {};
        if (MODE == 2) {                                       // dy, and scale P^T dy (threads 64-127)
            for (int i = tid; i < C * CW; i += NT) Y[(i % CW) * CP + i / CW] = V[i];
            __syncthreads();
            if (hi) tile<4>(F + (C + 4 * tr) * CP, CP, Y + tc * CP, 8 * CP, C, acc);
            else tile<4>(K + 4 * tr * L.ld, L.ld, S + tc * L.ld, 8 * L.ld, a.dk, acc);
            if (hi) {
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) W[(tc + 8 * c) * CP + 4 * tr + m] = a.scale * acc[m][c];
            }
            __syncthreads();
            if (!hi) {                                         // x
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 4 * tr + m;
                        acc[m][c] = fmaf(hh[t], acc[m][c], W[(tc + 8 * c) * CP + t]);
                        U[(tc + 8 * c) * CP + t] = be[t] * acc[m][c];
                    }
            }
            __syncthreads();
            if (!hi) {                                         // d; N is strictly lower, its transpose upper
                tile<4>(F + 4 * tr * CP, CP, U + tc * CP, 8 * CP, C, acc);
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 4 * tr + m, col = col0 + tc + 8 * c;
                        W[(tc + 8 * c) * CP + t] = -be[t] * g[t] * acc[m][c];
                        if (t < n && col < a.dv) {
                            y[vb + (t0 + t) * vs + col] = be[t] * acc[m][c];
                            r.rows[(chain * a.T + t0 + t) * a.dv + col] = acc[m][c];
                        }
                    }
            } else {                                           // scale g dy
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 4 * tr + m;
                        Y[(tc + 8 * c) * CP + t] *= a.scale * g[t];
                    }
            }
            __syncthreads();
        } else {
            if (MODE == 0 || !hi) tile<4>(K + (C * hi + 4 * tr) * L.ld, L.ld, S + tc * L.ld, 8 * L.ld, a.dk, acc);   // K S, Q S
            if (!hi) {
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 4 * tr + m;
                        acc[m][c] = t < n ? V[t * CW + tc + 8 * c] - g[t] * acc[m][c] : 0.f;
                        U[(tc + 8 * c) * CP + t] = be[t] * acc[m][c];
                    }
            }
            __syncthreads();
            if (!hi) {                                         // e
                tile<4>(F + 4 * tr * CP, CP, U + tc * CP, 8 * CP, 4 * tr + 4, acc);
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 4 * tr + m, col = col0 + tc + 8 * c;
                        const float w = be[t] * acc[m][c];
                        W[(tc + 8 * c) * CP + t] = hh[t] * w;
                        if (MODE == 0) Y[(tc + 8 * c) * CP + t] = w;
                        if (MODE == 1 && t < n && col < a.dv) r.rows[(chain * a.T + t0 + t) * a.dv + col] = acc[m][c];
                    }
            }
            __syncthreads();
            if (MODE == 0 && hi) {
                tile<4>(F + (C + 4 * tr) * CP, CP, Y + tc * CP, 8 * CP, 4 * tr + 4, out);
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int t = 4 * tr + m, col = col0 + tc + 8 * c;
                        if (t < n && col < a.dv) y[vb + (t0 + t) * vs + col] = a.scale * fmaf(g[t], acc[m][c], out[m][c]);
                    }
            }
            if (MODE == 0) __syncthreads();                    // Q S is out of S
        }
        // S[c][x] = g_31 S + sum_t (h w)[c][t] K[t][x]: four x and two columns a thread
        const float gl = g[C - 1];
        for (int p = tid; p < a.dk * 2; p += NT) {             // dk / 4 quads x 8 column pairs
            const int x = (p >> 3) * 4, c = p & 7;
            float4 s0 = *reinterpret_cast<const float4*>(S + c * L.ld + x), s1 = *reinterpret_cast<const float4*>(S + (c + 8) * L.ld + x);
            s0.x *= gl; s0.y *= gl; s0.z *= gl; s0.w *= gl;
            s1.x *= gl; s1.y *= gl; s1.z *= gl; s1.w *= gl;
#pragma unroll
            for (int pass = 0; pass < (MODE == 2 ? 2 : 1); ++pass) {
                const float* const A = K + pass * C * L.ld + x;
                const float* const B0 = (pass ? Y : W) + c * CP;
#pragma unroll 4
                for (int t = 0; t < C; t += 4) {
                    const float4 w0 = *reinterpret_cast<const float4*>(B0 + t), w1 = *reinterpret_cast<const float4*>(B0 + 8 * CP + t);
                    const float a0[4] = {w0.x, w0.y, w0.z, w0.w}, a1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 k = *reinterpret_cast<const float4*>(A + (t + e) * L.ld);
                        s0.x = fmaf(a0[e], k.x, s0.x); s0.y = fmaf(a0[e], k.y, s0.y); s0.z = fmaf(a0[e], k.z, s0.z); s0.w = fmaf(a0[e], k.w, s0.w);
                        s1.x = fmaf(a1[e], k.x, s1.x); s1.y = fmaf(a1[e], k.y, s1.y); s1.z = fmaf(a1[e], k.z, s1.z); s1.w = fmaf(a1[e], k.w, s1.w);
                    }
                }
            }
            *reinterpret_cast<float4*>(S + c * L.ld + x) = s0;
            *reinterpret_cast<float4*>(S + (c + 8) * L.ld + x) = s1;
        }
    }
    __syncthreads();
    if (MODE == 0 && chunks > 0) save(r.state + chain * per);
    if (MODE == 2 && r.state_out != nullptr) save(r.state_out + chain * per);
    if (MODE != 1)                                             // tokens past the length
        for (int t = len + tid / CW; t < a.T; t += NT / CW)
            if (col0 + tid % CW < a.dv) y[vb + t * vs + col0 + tid % CW] = 0.f;
}

template <int MODE>
cudaError_t walk(const GdnRecur& r, const float* fact, cudaStream_t stream) {
    const size_t smem = static_cast<size_t>(WalkLayout(r.a.dk).floats) * 4;
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_gdn_walk<MODE>, static_cast<size_t>(WalkLayout(256).floats) * 4, seen);
    if (e != cudaSuccess) return e;
    k_gdn_walk<MODE><<<dim3((r.a.dv + CW - 1) / CW, r.a.H, r.a.B), NT, smem, stream>>>(r, fact);
    return cudaGetLastError();
}

}  // namespace

size_t gdn_walk_bytes(int64_t chunks) { return static_cast<size_t>(chunks) * FACT * 4; }

bool gdn_walk_supported(int dtype, int B, int H, int T, int dv) {
    // the rule: the token recurrence has 0.27 us a token whatever the width, up to its 8 warps an SM
    return dtype == SDM_F32 && T >= C && static_cast<int64_t>(B) * H * ((dv + CW - 1) / CW) <= 152 * 8;
}

cudaError_t launch_gdn_walk(int mode, const GdnRecur& r, float* fact, cudaStream_t stream) {
    const GdnArgs& a = r.a;
    const size_t smem = static_cast<size_t>(64 * (a.dk + 4) + C * CP + 2 * C) * 4;
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_gdn_factors32, static_cast<size_t>(64 * 260 + C * CP + 2 * C) * 4, seen);
    if (e != cudaSuccess) return e;
    k_gdn_factors32<<<dim3((a.T + C - 1) / C, a.H, a.B), NT, smem, stream>>>(a, fact, mode == 2);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return mode == 0 ? walk<0>(r, fact, stream) : mode == 1 ? walk<1>(r, fact, stream) : walk<2>(r, fact, stream);
}

}  // namespace sdm
