// Gated delta rule, gradients of q, k, alpha and beta in fp32, every chunk of 32 tokens on its own.
//
// With S the state before a chunk, D the gradient of the state after it, w = beta e, the decay
// products G_ij = prod_{j < l <= i} alpha_l, g_i = prod_{l <= i} alpha_l and h_j = prod_{l > j}
// alpha_l inside the chunk (dy scaled by `scale`):
//   dq_i = g_i S dy_i + sum_{j <= i} M_ij k_j,                          M_ij = G_ij <dy_i, w_j>
//   dk_j = h_j D w_j - beta_j g_j S d_j + sum_{i >= j} M_ij q_i
//          - sum_{i > j} A_ij k_i - sum_{i < j} A_ji k_i,               A_ij = beta_i G_ij <d_i, w_j>
//   dbeta_i = <d_i, e_i>
// and the gradient of alpha_t is the sum of the gradients of the products it is a factor of, each
// with that factor left out.  With the chunk's start as column -1 and its end as row C,
//   X_ij = <dy_i, w_j> q_i.k_j - beta_i <d_i, w_j> k_i.k_j,   X_{i,-1} = q_i.S dy_i - beta_i k_i.S d_i,
//   X_{C,j} = k_j.D w_j,   X_{C,-1} = <D, S>,
//   dalpha_t = sum_{j < t} (sum_{i >= t} prod_{t < l <= i} alpha_l X_ij) prod_{j < l < t} alpha_l,
// which a lane per column runs backwards in t: nothing is divided by alpha, so gates of zero are
// exact.
//
// A CTA owns one chunk of one key head and adds up the gradients of the value heads that share it,
// so no atomics are needed.  Columns of the states come in blocks of 32; a thread keeps the outputs
// of one token and every eighth row of d_k.  Bound by shared-memory reads of the products over d_v.
#include "gdn_internal.h"

namespace sdm {

namespace {

constexpr int C = GDN_C32;
constexpr int CB = 32;           // state columns per block
constexpr int CP = CB + 4;       // their padded row (fp32), free of conflicts for 16-byte reads
constexpr int NT = 256;

template <int DKP>
struct Smem {
    float k[C][DKP + 4], q[C][DKP + 4];
    float S[DKP][CP], E[DKP][CP];
    float y[C][CP], d[C][CP], w[C][CP];
    float kk[C][C + 1], qk[C][C + 1];
    float yw[C][C + 1], dw[C][C + 1];       // <dy_i, w_j>, <d_i, w_j>; then M and A
    float X[C + 1][C + 1], G[C][C + 1];     // X: column j at j + 1
    float al[C], be[C], g[C], h[C], db[C];
    float part[NT / 32];
};

__device__ __forceinline__ float dot4(const float* a, const float* b, float s) {
    const float4 x = *reinterpret_cast<const float4*>(a), y = *reinterpret_cast<const float4*>(b);
    return fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s))));
}
template <class D> __device__ __forceinline__ void put_elem(void* base, int64_t i, float f);
template <> __device__ __forceinline__ void put_elem<F32>(void* base, int64_t i, float f) { static_cast<float*>(base)[i] = f; }
template <> __device__ __forceinline__ void put_elem<BF16>(void* base, int64_t i, float f) {
    static_cast<__nv_bfloat16*>(base)[i] = __float2bfloat16_rn(f);
}

template <class D, int DKP>
__global__ void __launch_bounds__(NT) k_gdn_grads(const GdnGrads r) {
    constexpr int R = DKP / 8;                  // rows of d_k per thread
    extern __shared__ __align__(16) unsigned char raw[];
    Smem<DKP>& sm = *reinterpret_cast<Smem<DKP>*>(raw);
    const GdnArgs& a = r.a;
    const int tid = threadIdx.x, ti = tid >> 3, rr = tid & 7;    // token, first row
    const int b = blockIdx.z, hk = blockIdx.y, ch = blockIdx.x, t0 = ch * C;
    const int nc = (a.T + C - 1) / C, group = a.H / a.Hk;
    const int len = gdn_length(a, b);
    const int n = len - t0 < C ? (len > t0 ? len - t0 : 0) : C;  // live tokens of the chunk
    const int nt = a.T - t0 < C ? a.T - t0 : C;                  // tokens of the chunk
    const int64_t kb = gdn_base(a.token_major, b, hk, a.Hk, a.T, a.dk), ks = gdn_stride(a.token_major, a.Hk, a.dk);

    for (int i = tid; i < C * DKP; i += NT) {
        const int t = i / DKP, x = i % DKP;
        const bool on = t < n && x < a.dk;
        const int64_t o = kb + (t0 + t) * ks + x;
        sm.k[t][x] = on ? load_elem<D>(a.k, o) : 0.f;
        sm.q[t][x] = on ? load_elem<D>(a.q, o) : 0.f;
    }
    __syncthreads();
    for (int m = 0; m < C / 8; ++m) {
        const int j = rr + 8 * m;
        float s = 0.f, u = 0.f;
        for (int x = 0; x < DKP; x += 4) {
            s = dot4(&sm.k[ti][x], &sm.k[j][x], s);
            u = dot4(&sm.q[ti][x], &sm.k[j][x], u);
        }
        sm.kk[ti][j] = s;
        sm.qk[ti][j] = u;
    }

    float dq[R], dk[R];
#pragma unroll
    for (int m = 0; m < R; ++m) dq[m] = dk[m] = 0.f;

    for (int hv = 0; hv < group; ++hv) {
        const int h = hk * group + hv;
        const int64_t chain = static_cast<int64_t>(b) * a.H + h;
        const int64_t per = static_cast<int64_t>(a.dk) * a.dv;
        const int64_t vb = gdn_base(a.token_major, b, h, a.H, a.T, a.dv), vs = gdn_stride(a.token_major, a.H, a.dv);
        if (n == 0) {                                            // past the length: zero gate gradients
            if (tid < nt) {
                put_elem<D>(r.dalpha, chain * a.T + t0 + tid, 0.f);
                put_elem<D>(r.dbeta, chain * a.T + t0 + tid, 0.f);
            }
            continue;
        }
        __syncthreads();                                         // the last head's reads are done
        if (tid < C) {
            const bool on = tid < n;
            sm.al[tid] = on ? load_elem<D>(a.alpha, chain * a.T + t0 + tid) : 1.f;
            sm.be[tid] = on ? load_elem<D>(a.beta, chain * a.T + t0 + tid) : 0.f;
        }
        __syncthreads();
        if (tid < 32) {                                          // column tid of the decay products
            float p = 1.f, gg = 1.f;
            for (int i = 0; i < C; ++i) {
                if (i > tid) p *= sm.al[i];
                sm.G[i][tid] = i >= tid ? p : 0.f;
                if (i <= tid) gg *= sm.al[i];
            }
            sm.h[tid] = p;
            sm.g[tid] = gg;
        }
        float yS[R], dS[R], wE[R];
#pragma unroll
        for (int m = 0; m < R; ++m) yS[m] = dS[m] = wE[m] = 0.f;
        float yw[C / 8], dw[C / 8], db = 0.f, es = 0.f;
#pragma unroll
        for (int m = 0; m < C / 8; ++m) yw[m] = dw[m] = 0.f;
        for (int c0 = 0; c0 < a.dv; c0 += CB) {
            __syncthreads();
            const float* Sp = r.S + (chain * nc + ch) * per;
            const float* Ep = r.dE + (chain * nc + ch) * per;
#pragma unroll(DKP <= 128 ? 4 : 1)
            for (int i = 0; i < DKP * CB / 4 / NT; ++i) {        // four columns of a row (d_v is a multiple of 4)
                const int p = tid + i * NT, x = p / (CB / 4), c = p % (CB / 4) * 4;
                const bool on = x < a.dk && c0 + c < a.dv;
                const int64_t o = static_cast<int64_t>(x) * a.dv + c0 + c;
                const float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
                const float4 s = on ? __ldg(reinterpret_cast<const float4*>(Sp + o)) : z, e = on ? __ldg(reinterpret_cast<const float4*>(Ep + o)) : z;
                *reinterpret_cast<float4*>(&sm.S[x][c]) = s;
                *reinterpret_cast<float4*>(&sm.E[x][c]) = e;
                es = fmaf(s.x, e.x, fmaf(s.y, e.y, fmaf(s.z, e.z, fmaf(s.w, e.w, es))));
            }
            {
                const int t = tid / (CB / 4), c = tid % (CB / 4) * 4;          // 32 tokens x 8 quads: one each
                const bool on = t < n && c0 + c < a.dv;
                const int64_t o = (chain * a.T + t0 + t) * a.dv + c0 + c;
                const float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
                *reinterpret_cast<float4*>(&sm.d[t][c]) = on ? __ldg(reinterpret_cast<const float4*>(r.d + o)) : z;
                *reinterpret_cast<float4*>(&sm.w[t][c]) = on ? __ldg(reinterpret_cast<const float4*>(r.e + o)) : z;   // e until its product with d is taken
#pragma unroll
                for (int j = 0; j < 4; ++j) sm.y[t][c + j] = on ? a.scale * load_elem<D>(r.dy, vb + (t0 + t) * vs + c0 + c + j) : 0.f;
            }
            __syncthreads();
            {   // dbeta, then w = beta e; four columns of one token per thread
                float4* wp = reinterpret_cast<float4*>(&sm.w[ti][4 * rr]);
                db = dot4(&sm.d[ti][4 * rr], &sm.w[ti][4 * rr], db);
                const float be = sm.be[ti];
                const float4 e = *wp;
                *wp = make_float4(be * e.x, be * e.y, be * e.z, be * e.w);
            }
            __syncthreads();
#pragma unroll 2
            for (int c = 0; c < CB; c += 4) {
                const float4 y = *reinterpret_cast<const float4*>(&sm.y[ti][c]);
                const float4 d = *reinterpret_cast<const float4*>(&sm.d[ti][c]);
                const float4 w = *reinterpret_cast<const float4*>(&sm.w[ti][c]);
#pragma unroll
                for (int m = 0; m < R; ++m) {
                    const float4 s = *reinterpret_cast<const float4*>(&sm.S[rr + 8 * m][c]);
                    const float4 e = *reinterpret_cast<const float4*>(&sm.E[rr + 8 * m][c]);
                    yS[m] = fmaf(y.x, s.x, fmaf(y.y, s.y, fmaf(y.z, s.z, fmaf(y.w, s.w, yS[m]))));
                    dS[m] = fmaf(d.x, s.x, fmaf(d.y, s.y, fmaf(d.z, s.z, fmaf(d.w, s.w, dS[m]))));
                    wE[m] = fmaf(w.x, e.x, fmaf(w.y, e.y, fmaf(w.z, e.z, fmaf(w.w, e.w, wE[m]))));
                }
#pragma unroll
                for (int m = 0; m < C / 8; ++m) {
                    const float4 u = *reinterpret_cast<const float4*>(&sm.w[rr + 8 * m][c]);
                    yw[m] = fmaf(y.x, u.x, fmaf(y.y, u.y, fmaf(y.z, u.z, fmaf(y.w, u.w, yw[m]))));
                    dw[m] = fmaf(d.x, u.x, fmaf(d.y, u.y, fmaf(d.z, u.z, fmaf(d.w, u.w, dw[m]))));
                }
            }
        }
        // sums over the eight threads of a token, and <D, S> over the CTA
        float qy = 0.f, kd = 0.f, kw = 0.f;
#pragma unroll
        for (int m = 0; m < R; ++m) {
            const int x = rr + 8 * m;
            qy = fmaf(sm.q[ti][x], yS[m], qy);
            kd = fmaf(sm.k[ti][x], dS[m], kd);
            kw = fmaf(sm.k[ti][x], wE[m], kw);
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
            qy += __shfl_xor_sync(0xffffffffu, qy, o);
            kd += __shfl_xor_sync(0xffffffffu, kd, o);
            kw += __shfl_xor_sync(0xffffffffu, kw, o);
            db += __shfl_xor_sync(0xffffffffu, db, o);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) es += __shfl_xor_sync(0xffffffffu, es, o);
        if ((tid & 31) == 0) sm.part[tid >> 5] = es;
        if (rr == 0) {
            sm.X[ti][0] = qy - sm.be[ti] * kd;
            sm.X[C][ti + 1] = kw;
            sm.db[ti] = db;
        }
#pragma unroll
        for (int m = 0; m < C / 8; ++m) {
            const int j = rr + 8 * m;
            const float be = sm.be[ti], G = sm.G[ti][j];
            const float u = ti >= j ? yw[m] : 0.f, w = ti > j ? be * dw[m] : 0.f;
            sm.X[ti][j + 1] = u * sm.qk[ti][j] - w * sm.kk[ti][j];
            sm.yw[ti][j] = G * u;
            sm.dw[ti][j] = G * w;
        }
        __syncthreads();
        if (tid == 0) {
            float s = 0.f;
            for (int i = 0; i < NT / 32; ++i) s += sm.part[i];
            sm.X[C][0] = s;
        }
        // intra-chunk products, then this head's share of the gradients
        const float gi = sm.g[ti], hi = sm.h[ti], bg = sm.be[ti] * sm.g[ti];
#pragma unroll
        for (int m = 0; m < R; ++m) {
            dq[m] = fmaf(gi, yS[m], dq[m]);
            dk[m] += hi * wE[m] - bg * dS[m];
        }
        for (int j = 0; j < C; ++j) {
            const float mij = sm.yw[ti][j], mji = sm.yw[j][ti];  // zero above the diagonal
            const float aij = sm.dw[ti][j] + sm.dw[j][ti];
#pragma unroll
            for (int m = 0; m < R; ++m) {
                const float kx = sm.k[j][rr + 8 * m], qx = sm.q[j][rr + 8 * m];
                dq[m] = fmaf(mij, kx, dq[m]);
                dk[m] = fmaf(mji, qx, fmaf(-aij, kx, dk[m]));
            }
        }
        __syncthreads();                                         // X[C][0]
        if (tid < 32) {
            // lane l walks column l - 1 (the start for l = 0), in place and eight rows at a time; column C - 1 has no
            // factor to its right inside the chunk, so it gives nothing.  Then lane t sums row t.
            float acc = sm.X[C][tid], next = 1.f;
#pragma unroll
            for (int q = C / 8 - 1; q >= 0; --q) {
                float v[8], al[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = sm.X[8 * q + e][tid];
                    al[e] = sm.al[8 * q + e];
                }
#pragma unroll
                for (int e = 7; e >= 0; --e) {
                    acc = fmaf(next, acc, v[e]);
                    next = al[e];
                    sm.X[8 * q + e][tid] = acc;
                }
            }
            float p = 1.f;                                       // prod_{j < l < t} alpha_l
#pragma unroll
            for (int q = 0; q < C / 8; ++q) {
                float v[8], al[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = sm.X[8 * q + e][tid];
                    al[e] = sm.al[8 * q + e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool on = 8 * q + e >= tid;
                    sm.X[8 * q + e][tid] = on ? v[e] * p : 0.f;
                    if (on) p *= al[e];
                }
            }
            __syncwarp();
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < C; ++j) s += sm.X[tid][j];
            if (tid < nt) {
                put_elem<D>(r.dalpha, chain * a.T + t0 + tid, tid < n ? s : 0.f);
                put_elem<D>(r.dbeta, chain * a.T + t0 + tid, tid < n ? sm.db[tid] : 0.f);
            }
        }
    }
    if (ti < nt) {
#pragma unroll
        for (int m = 0; m < R; ++m) {
            const int x = rr + 8 * m;
            if (x < a.dk) {
                put_elem<D>(r.dq, kb + (t0 + ti) * ks + x, ti < n ? dq[m] : 0.f);
                put_elem<D>(r.dk, kb + (t0 + ti) * ks + x, ti < n ? dk[m] : 0.f);
            }
        }
    }
}

template <class D, int DKP>
cudaError_t launch_one(const GdnGrads& g, cudaStream_t stream) {
    const size_t smem = sizeof(Smem<DKP>);
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_gdn_grads<D, DKP>, smem, seen);
    if (e != cudaSuccess) return e;
    const dim3 grid((g.a.T + C - 1) / C, g.a.Hk, g.a.B);
    k_gdn_grads<D, DKP><<<grid, NT, smem, stream>>>(g);
    return cudaGetLastError();
}

template <class D>
cudaError_t launch_rows(const GdnGrads& g, cudaStream_t stream) {
    if (g.a.dk <= 32) return launch_one<D, 32>(g, stream);
    if (g.a.dk <= 64) return launch_one<D, 64>(g, stream);
    if (g.a.dk <= 128) return launch_one<D, 128>(g, stream);
    return launch_one<D, 256>(g, stream);
}

}  // namespace

cudaError_t launch_gdn_grads(int dtype, const GdnGrads& g, cudaStream_t stream) {
    return dtype == SDM_F32 ? launch_rows<F32>(g, stream) : launch_rows<BF16>(g, stream);
}

}  // namespace sdm
