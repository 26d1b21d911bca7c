// Gated delta rule, token by token, in fp32 (every dtype, d_k <= 256, any d_v).
//
//   forward, per token:   S~ = alpha S;  e = v - S~^T k;  S = S~ + beta k e^T;  y = scale S^T q
//   reverse, per token:   D += scale q dy^T;  d = D^T k;  dv = beta d;  D = alpha (D - beta k d^T)
//
// Columns of the state never meet, so a warp owns 16 of them for the whole call and keeps its
// [d_k, 16] slice in registers: lane = 4 g + c holds columns 4c..4c+3 of the rows whose quad index
// is g modulo 8.  A quad of rows of k (or q) is one 8- or 16-byte shared-memory read that the four
// lanes of a group share, and the eight groups read neighbouring quads, so the reads are free of
// bank conflicts; rows are paired in the packed fp32x2 units.  The dot products over d_k end in
// three butterfly steps over the groups.  Blocks of TB tokens of q, k and v come through a
// double-buffered cp.async ring shared by the warps of the CTA.
//
// Bound by the latency of the chain, about 0.27 us a token up to two CTAs an SM.  A single token has a kernel of its own,
// k_gdn_step, below.
#include "gdn_internal.h"

namespace sdm {

namespace {

constexpr int TB = 16;          // tokens per staged block; divides the chunk lengths
constexpr int MAX_WARPS = 8;

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
          "l"(reinterpret_cast<unsigned long long&>(c)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return d;
}

__device__ __forceinline__ void cp16(void* dst, const void* src, bool on) {
    const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(dst));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(s), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

// Four consecutive storage elements of shared memory as two fp32 pairs.
template <class D> __device__ __forceinline__ void quad(const typename D::T* p, float2& a, float2& b);
template <> __device__ __forceinline__ void quad<F32>(const float* p, float2& a, float2& b) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    a = make_float2(f.x, f.y);
    b = make_float2(f.z, f.w);
}
template <> __device__ __forceinline__ void quad<BF16>(const __nv_bfloat16* p, float2& a, float2& b) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    a = make_float2(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u));
    b = make_float2(__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}
template <class D> __device__ __forceinline__ void put4(typename D::T* p, const float (&f)[4]);
template <> __device__ __forceinline__ void put4<F32>(float* p, const float (&f)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
template <> __device__ __forceinline__ void put4<BF16>(__nv_bfloat16* p, const float (&f)[4]) {
    __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}

// Sum of four columns over the eight row groups, in every lane.
__device__ __forceinline__ void sum_groups(float (&f)[4]) {
#pragma unroll
    for (int m = 4; m < 32; m <<= 1) {
#pragma unroll
        for (int c = 0; c < 4; ++c) f[c] += __shfl_xor_sync(0xffffffffu, f[c], m);
    }
}

template <class D, int Q>
struct Smem {
    typename D::T k[2][TB][32 * Q];
    typename D::T q[2][TB][32 * Q];
    typename D::T v[2][TB][16 * MAX_WARPS];     // v, or dy in reverse
    float a[2][TB], b[2][TB];
};

// MODE 0: forward; 1: forward with saved states; 2: reverse.  Grid (column blocks, H, B).
template <class D, int Q, int MODE>
__global__ void __launch_bounds__(32 * MAX_WARPS) k_gdn_recur(const GdnRecur r) {
    using T = typename D::T;
    extern __shared__ __align__(16) unsigned char raw[];
    Smem<D, Q>& sm = *reinterpret_cast<Smem<D, Q>*>(raw);
    const GdnArgs& a = r.a;
    const int b = blockIdx.z, h = blockIdx.y, hk = h / (a.H / a.Hk);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = (lane & 3) * 4;
    const int cols = static_cast<int>(blockDim.x >> 5) * 16;     // columns of this CTA
    const int col0 = blockIdx.x * cols, col = col0 + warp * 16 + c4;
    const bool live = col < a.dv;                                // d_v is a multiple of 4
    const int len = gdn_length(a, b);
    const int64_t chain = static_cast<int64_t>(b) * a.H + h;
    const int64_t vb = gdn_base(a.token_major, b, h, a.H, a.T, a.dv), vs = gdn_stride(a.token_major, a.H, a.dv);
    const int64_t kb = gdn_base(a.token_major, b, hk, a.Hk, a.T, a.dk), ks = gdn_stride(a.token_major, a.Hk, a.dk);
    T* y = static_cast<T*>(r.y);

    const int64_t per = static_cast<int64_t>(a.dk) * a.dv;
    const int64_t soff = chain * per;

    const int n = len;
    if (MODE != 1 && live && g == 0) {                            // tokens past the length
        const float z[4] = {0.f, 0.f, 0.f, 0.f};
        for (int t = n; t < a.T; ++t) put4<D>(y + vb + t * vs + col, z);
    }

    float2 S[2 * Q][4];      // [row pair][column]: rows 4 (8 i + g) + 2 p, + 1 for pair 2 i + p
    {
        const float* src = MODE == 0 ? r.state + soff : (r.state_in ? r.state_in + chain * per : nullptr);
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            float4 f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int rw = 4 * (8 * i + g) + j;
                f[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (src != nullptr && live && rw < a.dk)
                    f[j] = __ldcs(reinterpret_cast<const float4*>(src + static_cast<int64_t>(rw) * a.dv + col));
            }
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                S[2 * i + p][0] = make_float2(f[2 * p].x, f[2 * p + 1].x);
                S[2 * i + p][1] = make_float2(f[2 * p].y, f[2 * p + 1].y);
                S[2 * i + p][2] = make_float2(f[2 * p].z, f[2 * p + 1].z);
                S[2 * i + p][3] = make_float2(f[2 * p].w, f[2 * p + 1].w);
            }
        }
    }
    auto save = [&](float* dst) {
        if (!live) return;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int rw = 4 * (8 * i + g) + j, p = 2 * i + (j >> 1);
                if (rw < a.dk) {
                    const bool o = j & 1;
                    __stcs(reinterpret_cast<float4*>(dst + static_cast<int64_t>(rw) * a.dv + col),
                           make_float4(o ? S[p][0].y : S[p][0].x, o ? S[p][1].y : S[p][1].x,
                                       o ? S[p][2].y : S[p][2].x, o ? S[p][3].y : S[p][3].x));
                }
            }
        }
    };

    const int nblk = (n + TB - 1) / TB;
    const T* kp = static_cast<const T*>(a.k) + kb;
    const T* qp = static_cast<const T*>(a.q) + kb;
    const T* vp = static_cast<const T*>(MODE == 2 ? r.dy : a.v) + vb;
    auto stage = [&](int blk, int buf) {
        const int t0 = blk * TB;
        constexpr int KV = 32 * Q / D::E;                        // 16-byte pieces of a key row
        for (int i = threadIdx.x; i < TB * KV; i += blockDim.x) {
            const int t = i / KV, x = (i % KV) * D::E;
            const bool on = t0 + t < n && x < a.dk;              // d_k is a multiple of a piece
            const int64_t o = on ? (t0 + t) * ks + x : 0;
            cp16(&sm.k[buf][t][x], kp + o, on);
            if (MODE != 1) cp16(&sm.q[buf][t][x], qp + o, on);
        }
        const int VV = cols / D::E;
        for (int i = threadIdx.x; i < TB * VV; i += blockDim.x) {
            const int t = i / VV, x = (i % VV) * D::E;
            const bool on = t0 + t < n && col0 + x < a.dv;
            cp16(&sm.v[buf][t][x], vp + (on ? (t0 + t) * vs + col0 + x : 0), on);
        }
        cp_commit();
        if (threadIdx.x < TB) {
            const int t = t0 + threadIdx.x;
            sm.a[buf][threadIdx.x] = t < n ? load_elem<D>(a.alpha, chain * a.T + t) : 1.f;
            sm.b[buf][threadIdx.x] = t < n ? load_elem<D>(a.beta, chain * a.T + t) : 0.f;
        }
    };
    const int nc = (a.T + GDN_C32 - 1) / GDN_C32;
    constexpr int UN = Q <= 2 ? 4 : 2;
    auto block_of = [&](int i) { return MODE == 2 ? nblk - 1 - i : i; };
    if (nblk > 0) stage(block_of(0), 0);
    for (int i = 0; i < nblk; ++i) {
        const int buf = i & 1, blk = block_of(i), t0 = blk * TB;
        cp_wait<0>();
        __syncthreads();                                         // block i is in; block i - 1 is done with
        if (i + 1 < nblk) stage(block_of(i + 1), buf ^ 1);
        const int cnt = n - t0 < TB ? n - t0 : TB;
        if (MODE == 1 && t0 % GDN_C32 == 0) save(r.marks + (chain * nc + t0 / GDN_C32) * per);
        if (MODE == 2 && (t0 + cnt == n || (t0 + TB) % GDN_C32 == 0))
            save(r.marks + (chain * nc + t0 / GDN_C32) * per);
        auto token = [&](int j) {
            const int t = t0 + j;
            const float al = sm.a[buf][j], be = sm.b[buf][j];
            float2 va, vb2;
            quad<D>(&sm.v[buf][j][warp * 16 + c4], va, vb2);
            const float x[4] = {va.x, va.y, vb2.x, vb2.y};
            float2 k2[2 * Q];
#pragma unroll
            for (int p = 0; p < Q; ++p) quad<D>(&sm.k[buf][j][4 * (8 * p + g)], k2[2 * p], k2[2 * p + 1]);
            float2 acc[4];
            float s[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = make_float2(0.f, 0.f);
            if (MODE == 2) {
                float2 xs[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) xs[c] = make_float2(a.scale * x[c], a.scale * x[c]);
#pragma unroll
                for (int p = 0; p < Q; ++p) {
                    float2 q2[2];
                    quad<D>(&sm.q[buf][j][4 * (8 * p + g)], q2[0], q2[1]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        S[2 * p][c] = fma2(q2[0], xs[c], S[2 * p][c]);
                        S[2 * p + 1][c] = fma2(q2[1], xs[c], S[2 * p + 1][c]);
                    }
                }
            }
#pragma unroll
            for (int p = 0; p < 2 * Q; ++p) {
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[c] = fma2(k2[p], S[p][c], acc[c]);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) s[c] = acc[c].x + acc[c].y;
            sum_groups(s);
            const float2 al2 = make_float2(al, al);
            if (MODE == 2) {
                float o[4];
                float2 w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    o[c] = be * s[c];
                    w[c] = make_float2(-al * o[c], -al * o[c]);
                }
#pragma unroll
                for (int p = 0; p < 2 * Q; ++p) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) S[p][c] = fma2(k2[p], w[c], mul2(al2, S[p][c]));
                }
                if (live && g == 0) {
                    put4<D>(y + vb + t * vs + col, o);
                    put4<F32>(r.rows + (chain * a.T + t) * a.dv + col, s);
                }
            } else {
                float2 w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    s[c] = x[c] - al * s[c];                     // e
                    w[c] = make_float2(be * s[c], be * s[c]);
                }
                if (MODE == 1 && live && g == 0) put4<F32>(r.rows + (chain * a.T + t) * a.dv + col, s);
#pragma unroll
                for (int p = 0; p < 2 * Q; ++p) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) S[p][c] = fma2(k2[p], w[c], mul2(al2, S[p][c]));
                }
                if (MODE == 0) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[c] = make_float2(0.f, 0.f);
#pragma unroll
                    for (int p = 0; p < Q; ++p) {
                        float2 q2[2];
                        quad<D>(&sm.q[buf][j][4 * (8 * p + g)], q2[0], q2[1]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            acc[c] = fma2(q2[0], S[2 * p][c], acc[c]);
                            acc[c] = fma2(q2[1], S[2 * p + 1][c], acc[c]);
                        }
                    }
                    float o[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[c] = acc[c].x + acc[c].y;
                    sum_groups(o);
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[c] *= a.scale;
                    if (live && g == 0) put4<D>(y + vb + t * vs + col, o);
                }
            }
        };
        // whole blocks unrolled, so that the next tokens' reads and this one's output leave the chain
        if (cnt == TB) {
#pragma unroll UN
            for (int u = 0; u < TB; ++u) token(MODE == 2 ? TB - 1 - u : u);
        } else {
#pragma unroll 1
            for (int u = 0; u < cnt; ++u) token(MODE == 2 ? cnt - 1 - u : u);
        }
    }
    if (MODE == 0 && n > 0) save(r.state + soff);
    if (MODE == 2 && r.state_out != nullptr) save(r.state_out + chain * per);
}

// One token: the state's two trips through HBM are all that counts.  A CTA takes 32 columns of one state,
// a warp 32 rows of them, a lane 8 rows x 4 columns (a warp's load is four whole 128-byte row pieces), all
// in flight before anything is waited for but the slot.  Sums over d_k: two butterfly steps, then the warps'
// shares through shared memory.  At B = 256, H = 16, d_k = d_v = 128 the kernel above, with its staging and
// 1,420 instructions a warp, took 145 us for 541 MB; this one takes 84, 0.95 of the rate of a plain copy.
template <class D>
__device__ __forceinline__ void load8(const void* base, int64_t at, int left, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += D::E) {
        const uint4 u = left > i ? __ldg(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(base) + at + i)) : make_uint4(0, 0, 0, 0);
        unpack16<D>(u, f + i);
    }
}
template <class D> __device__ __forceinline__ void load4(const void* base, int64_t at, float (&f)[4]);
template <> __device__ __forceinline__ void load4<F32>(const void* base, int64_t at, float (&f)[4]) {
    const float4 u = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(base) + at));
    f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w;
}
template <> __device__ __forceinline__ void load4<BF16>(const void* base, int64_t at, float (&f)[4]) {
    const uint2 u = __ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(base) + at));
    f[0] = __uint_as_float(u.x << 16); f[1] = __uint_as_float(u.x & 0xffff0000u);
    f[2] = __uint_as_float(u.y << 16); f[3] = __uint_as_float(u.y & 0xffff0000u);
}

// Sum over the rows of the CTA of four columns per lane; `sh`: [warps][32 columns].
__device__ __forceinline__ void sum_rows(float (&f)[4], float (*sh)[32], int warp, int warps, int lane) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        f[c] += __shfl_xor_sync(0xffffffffu, f[c], 8);
        f[c] += __shfl_xor_sync(0xffffffffu, f[c], 16);
    }
    if (warps == 1) return;
    float4* const at = reinterpret_cast<float4*>(&sh[0][4 * (lane & 7)]);
    if (lane < 8) at[warp * 8] = make_float4(f[0], f[1], f[2], f[3]);
    __syncthreads();
    f[0] = f[1] = f[2] = f[3] = 0.f;
    for (int w = 0; w < warps; ++w) {
        const float4 o = at[w * 8];
        f[0] += o.x; f[1] += o.y; f[2] += o.z; f[3] += o.w;
    }
}

template <class D>
__global__ void __launch_bounds__(256) k_gdn_step(const GdnRecur r) {
    __shared__ __align__(16) float sh[2][8][32];
    const GdnArgs& a = r.a;
    const int b = blockIdx.z, h = blockIdx.y, hk = h / (a.H / a.Hk);
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const int row0 = 32 * warp + 8 * (lane >> 3), col = 32 * blockIdx.x + 4 * (lane & 7);
    const bool live = col < a.dv;                                // d_v is a multiple of 4
    int64_t slot = b;
    bool skip = gdn_length(a, b) == 0;
    if (r.slots != nullptr) {
        slot = __ldg(r.slots + b);
        if (slot >= r.n_slots && threadIdx.x == 0) flag_error(a.err, ERR_BAD_INDEX);
        skip = skip || slot < 0 || slot >= r.n_slots;
    }
    // with one token the two layouts are the same
    const int64_t chain = static_cast<int64_t>(b) * a.H + h, kb = (static_cast<int64_t>(b) * a.Hk + hk) * a.dk;
    float* const st = r.state + (slot * a.H + h) * a.dk * a.dv + col;
    const int left = a.dk - row0;                                // rows of this lane: 8, 4 or none of d_k's end
    float4 S[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        S[i] = !skip && live && i < left ? __ldcs(reinterpret_cast<const float4*>(st + static_cast<int64_t>(row0 + i) * a.dv)) : make_float4(0.f, 0.f, 0.f, 0.f);
    float k[8], q[8], v[4] = {0.f, 0.f, 0.f, 0.f};
    load8<D>(a.k, kb + row0, left, k);
    load8<D>(a.q, kb + row0, left, q);
    if (live) load4<D>(a.v, chain * a.dv + col, v);
    const float al = load_elem<D>(a.alpha, chain), be = load_elem<D>(a.beta, chain);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        s[0] = fmaf(k[i], S[i].x, s[0]); s[1] = fmaf(k[i], S[i].y, s[1]);
        s[2] = fmaf(k[i], S[i].z, s[2]); s[3] = fmaf(k[i], S[i].w, s[3]);
    }
    sum_rows(s, sh[0], warp, warps, lane);
    float w[4], o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = be * (v[c] - al * s[c]);  // beta e
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        S[i].x = fmaf(k[i], w[0], al * S[i].x); S[i].y = fmaf(k[i], w[1], al * S[i].y);
        S[i].z = fmaf(k[i], w[2], al * S[i].z); S[i].w = fmaf(k[i], w[3], al * S[i].w);
        if (!skip && live && i < left) __stcs(reinterpret_cast<float4*>(st + static_cast<int64_t>(row0 + i) * a.dv), S[i]);
        o[0] = fmaf(q[i], S[i].x, o[0]); o[1] = fmaf(q[i], S[i].y, o[1]);
        o[2] = fmaf(q[i], S[i].z, o[2]); o[3] = fmaf(q[i], S[i].w, o[3]);
    }
    sum_rows(o, sh[1], warp, warps, lane);
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = skip ? 0.f : a.scale * o[c];
    if (warp == 0 && lane < 8 && live) put4<D>(static_cast<typename D::T*>(r.y) + chain * a.dv + col, o);
}

template <class D, int Q>
cudaError_t launch_mode(int mode, const GdnRecur& r, dim3 grid, int threads, cudaStream_t stream) {
    const size_t smem = sizeof(Smem<D, Q>);
    static std::atomic<unsigned long long> seen[3];
    auto go = [&](auto kern) {
        cudaError_t e = allow_smem(kern, smem, seen[mode]);
        if (e != cudaSuccess) return e;
        kern<<<grid, threads, smem, stream>>>(r);
        return cudaGetLastError();
    };
    if (mode == 0) return go(k_gdn_recur<D, Q, 0>);
    if (mode == 1) return go(k_gdn_recur<D, Q, 1>);
    return go(k_gdn_recur<D, Q, 2>);
}

template <class D>
cudaError_t launch_rows(int mode, const GdnRecur& r, dim3 grid, int threads, cudaStream_t stream) {
    if (r.a.dk <= 32) return launch_mode<D, 1>(mode, r, grid, threads, stream);
    if (r.a.dk <= 64) return launch_mode<D, 2>(mode, r, grid, threads, stream);
    if (r.a.dk <= 128) return launch_mode<D, 4>(mode, r, grid, threads, stream);
    return launch_mode<D, 8>(mode, r, grid, threads, stream);
}

}  // namespace

cudaError_t launch_gdn_recur(int dtype, int mode, const GdnRecur& r, cudaStream_t stream) {
    const GdnArgs& a = r.a;
    if (mode == 0 && a.T == 1) {
        const dim3 grid((a.dv + 31) / 32, a.H, a.B);
        const int threads = 32 * ((a.dk + 31) / 32);
        if (dtype == SDM_F32) k_gdn_step<F32><<<grid, threads, 0, stream>>>(r);
        else k_gdn_step<BF16><<<grid, threads, 0, stream>>>(r);
        return cudaGetLastError();
    }
    // The warps of a CTA share the staged keys; few chains are spread over more, smaller CTAs so
    // that every SM has one.
    const int warps = (a.dv + 15) / 16;
    int per = warps < MAX_WARPS ? warps : MAX_WARPS;
    while (per > 1 && static_cast<int64_t>(a.B) * a.H * ((warps + per - 1) / per) < 152) per = (per + 1) / 2;
    const dim3 grid((warps + per - 1) / per, a.H, a.B);
    return dtype == SDM_F32 ? launch_rows<F32>(mode, r, grid, 32 * per, stream)
                            : launch_rows<BF16>(mode, r, grid, 32 * per, stream);
}

}  // namespace sdm
