// Norms after and before a block, with its gate, residual scale and residual, in one pass over the rows:
//   u = gamma_post y / rms(y),  h = x + res_scale gate u,  z = gamma_pre h / rms(h),  rms(a)^2 = mean a^2 + eps,
// and their gradients.  With n = h / rms(h) of the stored h and n' = y / rms(y):
//   dx = dh + (dn - n mean(dn n)) / rms(h),  dn = gamma_pre dz;     du = dx res_scale gate;
//   dy = (dn' - n' mean(dn' n')) / rms(y),   dn' = gamma_post du;
//   dgamma_pre = sum dz n,  dgamma_post = sum du n',  dres_scale = sum dx gate u,  dgate = sum dx res_scale u.
// Sums over a row: TPR threads a row, butterflies within a warp, then the warps' shares through shared memory.
#include "dla_internal.h"
#include "sdm_common.cuh"

#include <type_traits>

namespace sdm {

namespace {

// Threads of a CTA: one row or, where a row takes fewer than 256, several.
__host__ __device__ constexpr int cta(int tpr) { return tpr < 256 ? 256 : tpr; }

template <class D>
__device__ __forceinline__ uint4 load16(const void* base, int64_t at) {
    return __ldcs(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(base) + at));
}
template <class D>
__device__ __forceinline__ void store16(void* base, int64_t at, const uint4& u) {
    *reinterpret_cast<uint4*>(static_cast<typename D::T*>(base) + at) = u;
}
template <class D>
__device__ __forceinline__ void vec(const float* p, int x, float (&f)[D::E]) {
#pragma unroll
    for (int e = 0; e < D::E; e += 4) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p + x + e));
        f[e] = a.x; f[e + 1] = a.y; f[e + 2] = a.z; f[e + 3] = a.w;
    }
}

// Sums of N values over the TPR threads of a row, the same in all of them; other rows' threads are not waited for.
// `sh`: two sets of the warps' shares, used in turn, so that a sum's shares do not meet the readers of the one before.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float (*sh)[16][2], int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    if (TPR == 32) return;
    const int warp = threadIdx.x >> 5, sub = warp / (TPR / 32), first = sub * (TPR / 32);
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) sh[turn][warp][i] = s[i];
    }
    asm volatile("bar.sync %0, %1;\n" ::"r"(sub + 1), "n"(TPR) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = 0.f;
#pragma unroll
        for (int j = 0; j < TPR / 32; ++j) s[i] += sh[turn][first + j][i];
    }
    turn ^= 1;
}

// TPR threads a row, VE values a thread in pieces of 16 bytes, cta(TPR) / TPR rows a CTA at once.
template <class D, int TPR, int VE>
__global__ void __launch_bounds__(cta(TPR)) k_block_norm(const BlockNorm a) {
    constexpr int E = D::E, V = VE / E, ROWS = cta(TPR) / TPR;
    __shared__ float sh[2][16][2];
    int turn = 0;
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const float inv = 1.f / static_cast<float>(a.D);
    const bool post = a.gamma_post != nullptr;
    for (int64_t m = static_cast<int64_t>(blockIdx.x) * ROWS + sub; m < a.M; m += static_cast<int64_t>(gridDim.x) * ROWS) {
        uint4 xu[V], yu[V], gu[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            xu[i] = yu[i] = gu[i] = make_uint4(0, 0, 0, 0);
            if (c < a.D) {
                xu[i] = load16<D>(a.x, m * a.D + c);
                if (a.y != nullptr) yu[i] = load16<D>(a.y, m * a.D + c);
                if (a.gate != nullptr) gu[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(a.gate) + (a.gate_rows == 1 ? m : m / a.gate_rows) * a.D + c));
            }
        }
        float r = 1.f;
        if (post) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float f[8];
                unpack16<D>(yu[i], f);
#pragma unroll
                for (int e = 0; e < E; ++e) s[0] = fmaf(f[e], f[e], s[0]);
            }
            row_sum<TPR>(s, sh, turn);
            r = rsqrtf(fmaf(s[0], inv, a.eps));
        }
        float s[1] = {0.f};
        float h[V][E];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            float x[8], y[8];
            unpack16<D>(xu[i], x);
            unpack16<D>(yu[i], y);
            if (c < a.D && a.y != nullptr) {
                if (post) {
                    float g[E];
                    vec<D>(a.gamma_post, c, g);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] = y[e] * r * g[e];
                }
                if (a.gate != nullptr) {
                    float g[8];
                    unpack16<D>(gu[i], g);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] *= g[e];
                }
                if (a.res_scale != nullptr) {
                    float g[E];
                    vec<D>(a.res_scale, c, g);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] *= g[e];
                }
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] += y[e];
                const uint4 u = pack16<D>(x);
                store16<D>(a.h, m * a.D + c, u);
                unpack16<D>(u, x);                           // the norm is of what is stored
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                h[i][e] = x[e];
                s[0] = fmaf(x[e], x[e], s[0]);
            }
        }
        if (a.z == nullptr) continue;
        row_sum<TPR>(s, sh, turn);
        r = rsqrtf(fmaf(s[0], inv, a.eps));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            if (c >= a.D) continue;
            float g[E];
            vec<D>(a.gamma_pre, c, g);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = h[i][e] * r * g[e];
            store16<D>(a.z, m * a.D + c, pack16<D>(g));
        }
    }
}

// The gradients.  The rows are cut into items: ranges of `span` rows that, where the gradient of a gate shared by several
// rows is wanted, end with the gate's rows (`spans` to each), else anywhere.  A group of TPR threads takes every so many'th
// item, its rows one by one.  Column sums stay in registers: dgate's over an item, the others' over all the
// group's items; the shares go to `ws` and are joined in order by k_join.
struct NormCut {
    int64_t rows, span, items;   // rows that an item does not leave: a gate's, or all
    int64_t spans;
    unsigned grid;
    int groups;                  // of all CTAs
    size_t gate_at, total;       // floats of `ws`: [3][groups][D], then [items][D] where a gate has several items
};

template <class D, int TPR, int VE>
__global__ void __launch_bounds__(cta(TPR)) k_block_norm_backward(const BlockNorm a, const NormCut cut) {
    constexpr int E = D::E, V = VE / E, ROWS = cta(TPR) / TPR;
    __shared__ float sh[2][16][2];
    int turn = 0;
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const float inv = 1.f / static_cast<float>(a.D);
    const bool post = a.gamma_post != nullptr, pre = a.dz != nullptr;
    float sp[V][E], so[V][E], ss[V][E], sg[V][E];            // dgamma_pre, dgamma_post, dres_scale, dgate
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) sp[i][e] = so[i][e] = ss[i][e] = 0.f;
    const int group = blockIdx.x * ROWS + sub;
    const bool shared_gate = a.dgate != nullptr && a.gate_rows > 1;
    for (int64_t it = group; it < cut.items; it += cut.groups) {
        const int64_t part = it / cut.spans, g0 = part * cut.rows;
        const int64_t first = g0 + (it - part * cut.spans) * cut.span;
        int64_t last = g0 + cut.rows < first + cut.span ? g0 + cut.rows : first + cut.span;
        last = last < a.M ? last : a.M;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) sg[i][e] = 0.f;
        for (int64_t m = first; m < last; ++m) {
            uint4 hu[V], yu[V], zu[V], du[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                hu[i] = yu[i] = zu[i] = du[i] = make_uint4(0, 0, 0, 0);
                if (c < a.D) {
                    if (pre) {
                        hu[i] = load16<D>(a.h, m * a.D + c);
                        zu[i] = load16<D>(a.dz, m * a.D + c);
                    }
                    if (a.y != nullptr) yu[i] = load16<D>(a.y, m * a.D + c);
                    if (a.dh != nullptr) du[i] = load16<D>(a.dh, m * a.D + c);
                }
            }
            float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};      // of h and of y: sum of squares; of dn h
            if (pre) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (lane + i * TPR) * E;
                    if (c >= a.D) continue;
                    float h[8], z[8], g[E];
                    unpack16<D>(hu[i], h);
                    unpack16<D>(zu[i], z);
                    vec<D>(a.gamma_pre, c, g);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        s[0] = fmaf(h[e], h[e], s[0]);
                        t[0] = fmaf(z[e] * g[e], h[e], t[0]);
                    }
                }
            }
            if (post) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float y[8];
                    unpack16<D>(yu[i], y);
#pragma unroll
                    for (int e = 0; e < E; ++e) s[1] = fmaf(y[e], y[e], s[1]);
                }
            }
            float all[2] = {s[0], t[0]};
            if (pre) row_sum<TPR>(all, sh, turn);
            const float rh = rsqrtf(fmaf(all[0], inv, a.eps)), ch = all[1] * rh * rh * inv;      // mean(dn n) rh = ch rh; n = h rh
            float ry = 1.f;
            float one[1] = {s[1]};
            if (post) {
                row_sum<TPR>(one, sh, turn);
                ry = rsqrtf(fmaf(one[0], inv, a.eps));
            }
            float dn[V][E];
            float d1[1] = {0.f};
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                float dx[8];
                unpack16<D>(du[i], dx);
                if (pre) {
                    float h[8], z[8], g[E];
                    unpack16<D>(hu[i], h);
                    unpack16<D>(zu[i], z);
                    vec<D>(a.gamma_pre, c, g);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        sp[i][e] = fmaf(z[e], h[e] * rh, sp[i][e]);
                        dx[e] += rh * (z[e] * g[e] - h[e] * ch);
                    }
                }
                store16<D>(a.dx, m * a.D + c, pack16<D>(dx));
                if (a.y == nullptr) continue;
                float y[8], rs[E], gp[E], ga[8];
                unpack16<D>(yu[i], y);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    rs[e] = gp[e] = ga[e] = 1.f;
                    y[e] *= ry;                              // n' (y itself without a norm)
                }
                if (a.res_scale != nullptr) vec<D>(a.res_scale, c, rs);
                if (post) vec<D>(a.gamma_post, c, gp);
                if (a.gate != nullptr)
                    unpack16<D>(__ldg(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(a.gate) + (a.gate_rows == 1 ? m : m / a.gate_rows) * a.D + c)), ga);
                float dg[8];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float xu = dx[e] * (y[e] * gp[e]);
                    ss[i][e] = fmaf(xu, ga[e], ss[i][e]);
                    dg[e] = xu * rs[e];
                    sg[i][e] += dg[e];
                    const float d = dx[e] * rs[e] * ga[e];
                    so[i][e] = fmaf(d, y[e], so[i][e]);
                    dn[i][e] = d * gp[e];
                    d1[0] = fmaf(dn[i][e], y[e], d1[0]);
                }
                if (a.dgate != nullptr && a.gate_rows == 1) store16<D>(a.dgate, m * a.D + c, pack16<D>(dg));
            }
            if (a.y == nullptr) continue;
            float mean = 0.f;
            if (post) {
                row_sum<TPR>(d1, sh, turn);
                mean = d1[0] * inv;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                float y[8], d[8];
                unpack16<D>(yu[i], y);
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = post ? ry * (dn[i][e] - y[e] * ry * mean) : dn[i][e];
                store16<D>(a.dy, m * a.D + c, pack16<D>(d));
            }
        }
        if (shared_gate) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                if (cut.spans == 1) {
                    float f[8];
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] = sg[i][e];
                    store16<D>(a.dgate, part * a.D + c, pack16<D>(f));
                } else {
                    float* const to = a.ws + cut.gate_at + it * a.D + c;
#pragma unroll
                    for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(to + e) = make_float4(sg[i][e], sg[i][e + 1], sg[i][e + 2], sg[i][e + 3]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (lane + i * TPR) * E;
        if (c >= a.D) continue;
        const int64_t at = static_cast<int64_t>(group) * a.D + c, next = static_cast<int64_t>(cut.groups) * a.D;
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            if (a.dgamma_pre != nullptr) *reinterpret_cast<float4*>(a.ws + at + e) = make_float4(sp[i][e], sp[i][e + 1], sp[i][e + 2], sp[i][e + 3]);
            if (a.dgamma_post != nullptr) *reinterpret_cast<float4*>(a.ws + next + at + e) = make_float4(so[i][e], so[i][e + 1], so[i][e + 2], so[i][e + 3]);
            if (a.dres_scale != nullptr) *reinterpret_cast<float4*>(a.ws + 2 * next + at + e) = make_float4(ss[i][e], ss[i][e + 1], ss[i][e + 2], ss[i][e + 3]);
        }
    }
}

// out[j][c] = sum over n rows of part[j][n][c], in order: 32 columns a CTA, eight ranges of rows.  With `each` the outputs
// lie one after the other in o0.
template <class D>
__global__ void __launch_bounds__(256) k_join(const float* __restrict__ part, int n, int width, void* o0, void* o1, void* o2, int64_t each) {
    __shared__ float sum[8][33];
    const int cols = (width + 31) / 32, j = blockIdx.x / cols;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x % cols * 32 + x;
    const float* p = part + j * static_cast<int64_t>(n) * width;
    void* out = each ? o0 : j == 0 ? o0 : j == 1 ? o1 : o2;
    if (out == nullptr) return;
    float s = 0.f;
    if (c < width)
        for (int i = y; i < n; i += 8) s += __ldcs(p + static_cast<int64_t>(i) * width + c);
    sum[y][x] = s;
    __syncthreads();
    if (y == 0 && c < width) {
        for (int i = 1; i < 8; ++i) s += sum[i][x];
        const int64_t at = j * each + c;
        if (D::BYTES == 4) static_cast<float*>(out)[at] = s;
        else static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(s);
    }
}

constexpr int SMS = 152;

// `shared`: the gradient of a gate shared by several rows is wanted.
NormCut norm_cut(int64_t M, int64_t gate_rows, int D, int rows, bool shared) {
    NormCut c{};
    c.rows = shared && gate_rows < M ? gate_rows : M;
    const int64_t parts = (M + c.rows - 1) / c.rows, want = static_cast<int64_t>(SMS) * 4 * rows;
    c.spans = (want + parts - 1) / parts;
    if (c.spans > c.rows) c.spans = c.rows;
    c.span = (c.rows + c.spans - 1) / c.spans;
    c.spans = (c.rows + c.span - 1) / c.span;
    c.items = parts * c.spans;
    const int64_t ctas = (c.items + rows - 1) / rows;
    c.grid = static_cast<unsigned>(ctas < SMS * 4 ? ctas : SMS * 4);
    c.groups = static_cast<int>(c.grid) * rows;
    c.gate_at = static_cast<size_t>(3) * c.groups * D;
    c.total = c.gate_at + (shared && c.spans > 1 ? static_cast<size_t>(c.items) * D : 0);
    return c;
}

// Threads a row and values a thread: eight values while a row has at most 512 threads of them.
struct RowPlan {
    int tpr, ve;
};
RowPlan row_plan(int D) {
    RowPlan p{32, 8};
    while (p.tpr < 512 && p.tpr * 8 < D) p.tpr *= 2;
    while (p.tpr * p.ve < D) p.ve *= 2;
    return p;
}

template <class F>
cudaError_t with_plan(const RowPlan& p, F f) {
#define SDM_ROW(T, V) if (p.tpr == T && p.ve == V) return f(std::integral_constant<int, T>{}, std::integral_constant<int, V>{});
    SDM_ROW(32, 8) SDM_ROW(64, 8) SDM_ROW(128, 8) SDM_ROW(256, 8) SDM_ROW(512, 8) SDM_ROW(512, 16) SDM_ROW(512, 32)
#undef SDM_ROW
    return cudaErrorInvalidValue;
}

template <class D>
cudaError_t forward(const RowPlan& p, const BlockNorm& a, cudaStream_t stream) {
    return with_plan(p, [&](auto T, auto V) {
        const int64_t rows = cta(T.value) / T.value, need = (a.M + rows - 1) / rows;
        const unsigned grid = static_cast<unsigned>(need < SMS * 8 ? need : SMS * 8);
        k_block_norm<D, T.value, V.value><<<grid, cta(T.value), 0, stream>>>(a);
        return cudaGetLastError();
    });
}
template <class D>
cudaError_t backward(const RowPlan& p, const BlockNorm& a, cudaStream_t stream) {
    const int rows = cta(p.tpr) / p.tpr;
    const bool shared = a.dgate != nullptr && a.gate_rows > 1;
    const NormCut cut = norm_cut(a.M, a.gate_rows, a.D, rows, shared);
    cudaError_t e = with_plan(p, [&](auto T, auto V) {
        k_block_norm_backward<D, T.value, V.value><<<cut.grid, cta(T.value), 0, stream>>>(a, cut);
        return cudaGetLastError();
    });
    const unsigned cols = static_cast<unsigned>((a.D + 31) / 32);
    if (e == cudaSuccess && (a.dgamma_pre != nullptr || a.dgamma_post != nullptr || a.dres_scale != nullptr)) {
        k_join<F32><<<3 * cols, 256, 0, stream>>>(a.ws, cut.groups, a.D, a.dgamma_pre, a.dgamma_post, a.dres_scale, 0);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess && shared && cut.spans > 1) {
        k_join<D><<<cols * static_cast<unsigned>(cut.items / cut.spans), 256, 0, stream>>>(a.ws + cut.gate_at, static_cast<int>(cut.spans), a.D, a.dgate, nullptr, nullptr, a.D);
        e = cudaGetLastError();
    }
    return e;
}

}  // namespace

bool block_norm_supported(int D) { return D <= 512 * 32; }
cudaError_t launch_block_norm(int dtype, const BlockNorm& a, cudaStream_t stream) {
    const RowPlan p = row_plan(a.D);
    return dtype == SDM_F32 ? forward<F32>(p, a, stream) : forward<BF16>(p, a, stream);
}
size_t block_norm_backward_bytes(int64_t M, int64_t gate_rows, int D) {
    if (M == 0) return 0;
    const int tpr = row_plan(D).tpr;
    const size_t one = norm_cut(M, gate_rows, D, cta(tpr) / tpr, false).total, each = norm_cut(M, gate_rows, D, cta(tpr) / tpr, gate_rows > 1).total;
    return (one > each ? one : each) * 4;
}
cudaError_t launch_block_norm_backward(int dtype, const BlockNorm& a, cudaStream_t stream) {
    const RowPlan p = row_plan(a.D);
    return dtype == SDM_F32 ? backward<F32>(p, a, stream) : backward<BF16>(p, a, stream);
}

}  // namespace sdm
