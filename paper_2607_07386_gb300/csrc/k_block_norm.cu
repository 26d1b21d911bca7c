// Norms after and before a block, with its gate, residual scale and residual, in one pass over the rows:
//   u = gamma_post y / rms(y),  h = x + res_scale gate u,  z = gamma_pre h / rms(h),  rms(a)^2 = mean a^2 + eps,
// and their gradients.  With n = h / rms(h) of the stored h, n' = y / rms(y) and c = res_scale gamma_post:
//   dx = dh + (dn - n mean(dn n)) / rms(h),  dn = gamma_pre dz;
//   dy = (dn' - n' mean(dn' n')) / rms(y),   dn' = dx gate c, whose mean follows from sums that need neither norm, so that
//   a row takes one reduction;
//   dgamma_pre = sum dz n;  with q = dx n':  dgate = c sum q over the gate's rows,
//   G = sum gate q over all:  dres_scale = gamma_post G,  dgamma_post = res_scale G.
// So two column sums are all that the gradients of four vectors take.  Sums over a row: TPR threads a row, butterflies
// within a warp, then the warps' shares through shared memory.
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
template <int E>
__device__ __forceinline__ void put_floats(float* to, const float (&f)[E]) {
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(to + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
}
template <class D>
__device__ __forceinline__ void vec(const float* p, int x, float (&f)[D::E]) {
#pragma unroll
    for (int e = 0; e < D::E; e += 4) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p + x + e));
        f[e] = a.x; f[e + 1] = a.y; f[e + 2] = a.z; f[e + 3] = a.w;
    }
}

// Sums of up to eight values over the TPR threads of a row, the same in all of them; other rows' threads are not waited
// for.  The lanes first halve the values they hold at every step (9 shuffles for eight values, 5 for one), then add up one each.
// `sh`: two sets of the warps' shares, used in turn, so that a sum's shares do not meet the readers of the one before.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float (*sh)[16][8], int& turn) {
    const int lane = threadIdx.x & 31;
    if (N == 1) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
        if (TPR == 32) return;
    }
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < N ? s[i] : 0.f;
    if (N > 1) {
#pragma unroll
        for (int o = 16, n = 4; n > 0; o >>= 1, n >>= 1) {
            const bool up = lane & o;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        }
        v[0] += __shfl_xor_sync(0xffffffffu, v[0], 2);
        v[0] += __shfl_xor_sync(0xffffffffu, v[0], 1);       // value lane / 4 of the eight
        if (TPR == 32) {
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = __shfl_sync(0xffffffffu, v[0], 4 * i);
            return;
        }
    }
    const int warp = threadIdx.x >> 5, sub = warp / (TPR / 32), first = sub * (TPR / 32);
    if (N == 1 ? lane == 0 : lane % 4 == 0) sh[turn][warp][lane / 4] = v[0];
    asm volatile("bar.sync %0, %1;\n" ::"r"(sub + 1), "n"(TPR) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < TPR / 32; ++j) {
        if (N == 1) {
            s[0] += sh[turn][first + j][0];
            continue;
        }
        const float4 x = *reinterpret_cast<const float4*>(sh[turn][first + j]), y = *reinterpret_cast<const float4*>(sh[turn][first + j] + 4);
        const float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += f[i];
    }
    turn ^= 1;
}

constexpr int SMS = 152, FORE_CTAS = 3, BACK_CTAS = 2;       // CTAs of 256 threads on an SM: 80 and 128 registers a thread

// Threads a row, values a thread in pieces of 16 bytes, rows of a CTA at once.
template <class D, int TPR, int VE>
struct Row {
    static constexpr int E = D::E, V = VE / E, ROWS = cta(TPR) / TPR;
    static constexpr bool KEEP = VE == 8;        // the vectors' values of a thread stay in registers
};
// The values at column c of a vector that may be missing (ones), times those of another.
template <class D>
__device__ __forceinline__ void ones_or(const float* p, int c, float (&f)[D::E]) {
    if (p != nullptr) {
        vec<D>(p, c, f);
    } else {
#pragma unroll
        for (int e = 0; e < D::E; ++e) f[e] = 1.f;
    }
}
template <class D>
__device__ __forceinline__ void product(const float* p, const float* q, int c, float (&f)[D::E]) {
    float g[D::E];
    ones_or<D>(p, c, f);
    ones_or<D>(q, c, g);
#pragma unroll
    for (int e = 0; e < D::E; ++e) f[e] *= g[e];
}

// Rows on their way: each thread copies its own pieces of N arrays' next S rows into slots of its own in shared memory
// (asynchronously, so no registers are held and nothing has to be waited for but its own copies).  With S = 0, where S
// rows of the widest type do not fit, rows are loaded when they are due.
template <class D, int TPR, int VE, int N, int S>
struct Ahead {
    using R = Row<D, TPR, VE>;
    static constexpr int SLOTS = S > 0 ? S : 1;
    uint4* const base;               // [S][N][V][threads]
    int64_t next, last;              // the next row to copy, and the end
    int D_;
    int at;                          // the slot of the row at hand
    __device__ __forceinline__ Ahead(unsigned char* smem, int64_t first, int64_t end, int D0)
        : base(reinterpret_cast<uint4*>(smem) + threadIdx.x), next(first), last(end), D_(D0), at(0) {}
    __device__ __forceinline__ uint4* slot(int s, int n, int i) const { return base + ((s * N + n) * R::V + i) * cta(TPR); }
    __device__ __forceinline__ void copy(int s, const void* const (&src)[N]) {
        if (next < last) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (src[n] == nullptr) continue;
#pragma unroll
                for (int i = 0; i < R::V; ++i) {
                    const int c = (static_cast<int>(threadIdx.x) % TPR + i * TPR) * R::E;
                    if (c < D_)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(slot(s, n, i)))),
                                     "l"(static_cast<const typename D::T*>(src[n]) + next * D_ + c) : "memory");
                }
            }
            ++next;
        }
        asm volatile("cp.async.commit_group;\n" ::: "memory");
    }
    __device__ __forceinline__ void start(const void* const (&src)[N]) {
#pragma unroll
        for (int s = 0; s < S; ++s) copy(s, src);
    }
    __device__ __forceinline__ void wait() {
        if (S > 0) asm volatile("cp.async.wait_group %0;\n" ::"n"(S > 0 ? S - 1 : 0) : "memory");
    }
    // Piece i of array n of row m; zeros behind the row's end and where there is no array.
    __device__ __forceinline__ uint4 get(const void* const (&src)[N], int64_t m, int n, int i) const {
        const int c = (static_cast<int>(threadIdx.x) % TPR + i * TPR) * R::E;
        if (c >= D_ || src[n] == nullptr) return make_uint4(0, 0, 0, 0);
        if (S == 0) return load16<D>(src[n], m * D_ + c);
        return *slot(at, n, i);
    }
    // The row at hand is done with.
    __device__ __forceinline__ void advance(const void* const (&src)[N]) {
        if (S == 0) return;
        copy(at, src);
        at = at + 1 == SLOTS ? 0 : at + 1;
    }
};

// A group of TPR threads takes `span` rows one after the other.
template <class D, int TPR, int VE, int S>
__global__ void __launch_bounds__(cta(TPR), TPR > 256 ? 1 : FORE_CTAS) k_block_norm(const BlockNorm a, const int64_t span) {
    extern __shared__ __align__(16) unsigned char ring[];
    using R = Row<D, TPR, VE>;
    constexpr int E = R::E, V = R::V;
    __shared__ __align__(16) float sh[2][16][8];
    int turn = 0;
    const int lane = threadIdx.x % TPR;
    const float inv = 1.f / static_cast<float>(a.D);
    const bool post = a.gamma_post != nullptr, has_y = a.y != nullptr, pre = a.z != nullptr;
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * R::ROWS + threadIdx.x / TPR) * span;
    const int64_t last = first + span < a.M ? first + span : a.M;
    if (first >= last) return;
    uint4 gu[V];
    const void* const src[2] = {a.x, a.y};
    Ahead<D, TPR, VE, 2, S> rows(ring, first, last, a.D);
    rows.start(src);
    auto gate = [&](int64_t g) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            gu[i] = c < a.D ? __ldg(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(a.gate) + g * a.D + c)) : make_uint4(0, 0, 0, 0);
        }
    };
    int64_t g = a.gate != nullptr ? first / a.gate_rows : 0, until = a.gate != nullptr ? (g + 1) * a.gate_rows : last;
    if (a.gate != nullptr) gate(g);
    float ck[R::KEEP ? V : 1][E], pk[R::KEEP ? V : 1][E];
    if (R::KEEP) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            if (c < a.D) {
                product<D>(a.res_scale, a.gamma_post, c, ck[i]);
                ones_or<D>(a.gamma_pre, c, pk[i]);
            }
        }
    }
    for (int64_t m = first; m < last; ++m) {
        uint4 xu[V], yu[V];
        rows.wait();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            xu[i] = rows.get(src, m, 0, i);
            yu[i] = rows.get(src, m, 1, i);
        }
        rows.advance(src);
        if (m == until) {
            gate(++g);
            until += a.gate_rows;
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
        if (has_y) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                float x[8], y[8], k[E], ga[8];
                unpack16<D>(xu[i], x);
                unpack16<D>(yu[i], y);
                if (a.gate != nullptr) unpack16<D>(gu[i], ga);
                if (!R::KEEP) product<D>(a.res_scale, a.gamma_post, c, k);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    y[e] = y[e] * r * (R::KEEP ? ck[i][e] : k[e]);
                    if (a.gate != nullptr) y[e] *= ga[e];
                    x[e] += y[e];
                }
                xu[i] = pack16<D>(x);
                store16<D>(a.h, m * a.D + c, xu[i]);
            }
        }
        if (!pre) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {                        // of what is stored
            float x[8];
            unpack16<D>(xu[i], x);
#pragma unroll
            for (int e = 0; e < E; ++e) s[0] = fmaf(x[e], x[e], s[0]);
        }
        row_sum<TPR>(s, sh, turn);
        r = rsqrtf(fmaf(s[0], inv, a.eps));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            if (c >= a.D) continue;
            float x[8], k[E];
            unpack16<D>(xu[i], x);
            if (!R::KEEP) vec<D>(a.gamma_pre, c, k);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = x[e] * r * (R::KEEP ? pk[i][e] : k[e]);
            store16<D>(a.z, m * a.D + c, pack16<D>(x));
        }
    }
}

// The gradients.  The rows are cut into items: ranges of `span` rows that, where the gradient of a gate shared by several
// rows is wanted, end with the gate's rows (`spans` to each), else anywhere.  A group of TPR threads takes every so many'th
// item, its rows one by one.  Column sums stay in registers: q's over an item, the others' over all the
// group's items; the shares go to `ws` and are joined in order.
struct NormCut {
    int64_t rows, span, items;   // rows that an item does not leave: a gate's, or all
    int64_t spans;
    unsigned grid;
    int groups;                  // of all CTAs
    size_t gate_at, total;       // floats of `ws`: [2][groups][D], then [items][D] where a gate has several items
};

template <class D, int TPR, int VE, int S>
__global__ void __launch_bounds__(cta(TPR), TPR > 256 ? 1 : BACK_CTAS) k_block_norm_backward(const BlockNorm a, const NormCut cut) {
    extern __shared__ __align__(16) unsigned char ring[];
    using R = Row<D, TPR, VE>;
    constexpr int E = R::E, V = R::V;
    __shared__ __align__(16) float sh[2][16][8];
    int turn = 0;
    const int lane = threadIdx.x % TPR, group = blockIdx.x * R::ROWS + threadIdx.x / TPR;
    const float inv = 1.f / static_cast<float>(a.D);
    const bool post = a.gamma_post != nullptr, pre = a.dz != nullptr, has_y = a.y != nullptr, has_gate = a.gate != nullptr;
    const bool shared_gate = a.dgate != nullptr && a.gate_rows > 1;
    float sp[V][E], sq[V][E], sG[V][E];                      // sums of dz n, of q, and G
    float ck[R::KEEP ? V : 1][E], pk[R::KEEP ? V : 1][E];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (lane + i * TPR) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) sp[i][e] = sG[i][e] = 0.f;
        if (R::KEEP && c < a.D) {
            product<D>(a.res_scale, a.gamma_post, c, ck[i]);
            ones_or<D>(a.gamma_pre, c, pk[i]);
        }
    }
    const void* const src[4] = {pre ? a.h : nullptr, a.dz, a.y, a.dh};
    for (int64_t it = group; it < cut.items; it += cut.groups) {
        const int64_t part = it / cut.spans, g0 = part * cut.rows;
        const int64_t first = g0 + (it - part * cut.spans) * cut.span;
        int64_t last = g0 + cut.rows < first + cut.span ? g0 + cut.rows : first + cut.span;
        last = last < a.M ? last : a.M;
        uint4 gu[V];
        int64_t g = -1, until = first;                       // the gate's row at hand, and its end
        auto gate = [&](int64_t m) {
            g = m / a.gate_rows;
            until = (g + 1) * a.gate_rows;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                gu[i] = c < a.D ? __ldg(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(a.gate) + g * a.D + c)) : make_uint4(0, 0, 0, 0);
            }
        };
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) sq[i][e] = 0.f;
        Ahead<D, TPR, VE, 4, S> rows(ring, first, last, a.D);
        rows.start(src);
        for (int64_t m = first; m < last; ++m) {
            uint4 hu[V], yu[V], zu[V], du[V];
            rows.wait();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                hu[i] = rows.get(src, m, 0, i);
                zu[i] = rows.get(src, m, 1, i);
                yu[i] = rows.get(src, m, 2, i);
                du[i] = rows.get(src, m, 3, i);
            }
            rows.advance(src);
            if (has_gate && m == until) gate(m);
            // sums of h^2, dn h, y^2 and, with b = gate c y, of b dh, b dn and b h
            float s[6] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                float h[8], z[8], y[8], d[8], ga[8], k[E], kc[E];
                unpack16<D>(hu[i], h);
                unpack16<D>(zu[i], z);
                unpack16<D>(yu[i], y);
                unpack16<D>(du[i], d);
                if (has_gate) unpack16<D>(gu[i], ga);
                if (!R::KEEP) ones_or<D>(a.gamma_pre, c, k);
                if (!R::KEEP) product<D>(a.res_scale, a.gamma_post, c, kc);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float n = z[e] * (R::KEEP ? pk[i][e] : k[e]);
                    float b = y[e] * (R::KEEP ? ck[i][e] : kc[e]);
                    if (has_gate) b *= ga[e];
                    s[0] = fmaf(h[e], h[e], s[0]);
                    s[1] = fmaf(n, h[e], s[1]);
                    s[2] = fmaf(y[e], y[e], s[2]);
                    s[3] = fmaf(b, d[e], s[3]);
                    s[4] = fmaf(b, n, s[4]);
                    s[5] = fmaf(b, h[e], s[5]);
                }
            }
            if (pre || post) row_sum<TPR>(s, sh, turn);
            const float rh = pre ? rsqrtf(fmaf(s[0], inv, a.eps)) : 0.f, ch = s[1] * rh * rh * inv;      // mean(dn n) rh = ch rh; n = h rh
            const float ry = post ? rsqrtf(fmaf(s[2], inv, a.eps)) : 1.f;
            // mean(dn' n') = ry mean(b dx), dx = dh + rh (dn - h ch)
            const float mean = post ? ry * inv * (pre ? s[3] + rh * (s[4] - ch * s[5]) : s[3]) : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                float dx[8], k[E];
                unpack16<D>(du[i], dx);
                if (pre) {
                    float h[8], z[8];
                    unpack16<D>(hu[i], h);
                    unpack16<D>(zu[i], z);
                    if (!R::KEEP) vec<D>(a.gamma_pre, c, k);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        sp[i][e] = fmaf(z[e], h[e] * rh, sp[i][e]);
                        dx[e] += rh * (z[e] * (R::KEEP ? pk[i][e] : k[e]) - h[e] * ch);
                    }
                }
                store16<D>(a.dx, m * a.D + c, pack16<D>(dx));
                if (!has_y) continue;
                float y[8], ga[8], dg[8];
                unpack16<D>(yu[i], y);
                if (has_gate) {
                    unpack16<D>(gu[i], ga);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) ga[e] = 1.f;
                }
                if (!R::KEEP) product<D>(a.res_scale, a.gamma_post, c, k);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float n = y[e] * ry, q = dx[e] * n, ce = R::KEEP ? ck[i][e] : k[e];       // n': y itself without a norm
                    if (shared_gate) sq[i][e] += q;
                    else sG[i][e] = fmaf(ga[e], q, sG[i][e]);
                    dg[e] = q * ce;
                    const float dn = dx[e] * ga[e] * ce;
                    dx[e] = post ? ry * (dn - n * mean) : dn;
                }
                if (a.dgate != nullptr && !shared_gate) store16<D>(a.dgate, m * a.D + c, pack16<D>(dg));
                store16<D>(a.dy, m * a.D + c, pack16<D>(dx));
            }
        }
        if (shared_gate) {
            if (first < last || cut.spans > 1) {
                if (first < last && g < 0) gate(first);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (lane + i * TPR) * E;
                    if (c >= a.D) continue;
                    float ga[8], f[8], k[E];
                    if (first < last) {
                        unpack16<D>(gu[i], ga);
#pragma unroll
                        for (int e = 0; e < E; ++e) sG[i][e] = fmaf(ga[e], sq[i][e], sG[i][e]);
                    }
                    if (cut.spans == 1) {
                        if (!R::KEEP) product<D>(a.res_scale, a.gamma_post, c, k);
#pragma unroll
                        for (int e = 0; e < E; ++e) f[e] = sq[i][e] * (R::KEEP ? ck[i][e] : k[e]);
                        store16<D>(a.dgate, part * a.D + c, pack16<D>(f));
                    } else {
                        put_floats<E>(a.ws + cut.gate_at + it * a.D + c, sq[i]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (lane + i * TPR) * E;
        if (c >= a.D) continue;
        float* const at = a.ws + static_cast<int64_t>(group) * a.D + c;
        if (a.dgamma_pre != nullptr) put_floats<E>(at, sp[i]);
        if (a.dgamma_post != nullptr || a.dres_scale != nullptr) put_floats<E>(at + static_cast<int64_t>(cut.groups) * a.D, sG[i]);
    }
}

// Sums over the shares, in order: JC columns a CTA, JR ranges of rows.  Job 0: dgamma_pre, 1: dres_scale and dgamma_post from
// G, 2 and on: the rows of dgate.
constexpr int JC = 8, JR = 32;
template <class D>
__global__ void __launch_bounds__(JC * JR) k_block_norm_join(const BlockNorm a, const NormCut cut) {
    __shared__ float sum[JR][JC + 1];
    const int cols = (a.D + JC - 1) / JC, job = blockIdx.x / cols;
    const int x = threadIdx.x % JC, y = threadIdx.x / JC, c = blockIdx.x % cols * JC + x;
    if (job == 0 ? a.dgamma_pre == nullptr : job == 1 && a.dgamma_post == nullptr && a.dres_scale == nullptr) return;
    const int64_t n = job < 2 ? cut.groups : cut.spans;
    const float* p = a.ws + (job < 2 ? static_cast<int64_t>(job) * cut.groups * a.D : cut.gate_at + (job - 2) * cut.spans * a.D);
    float s = 0.f;
    if (c < a.D)
#pragma unroll 4
        for (int64_t i = y; i < n; i += JR) s += __ldcs(p + i * a.D + c);
    sum[y][x] = s;
    __syncthreads();
    if (y != 0 || c >= a.D) return;
    for (int i = 1; i < JR; ++i) s += sum[i][x];
    if (job == 0) {
        a.dgamma_pre[c] = s;
    } else if (job == 1) {
        if (a.dres_scale != nullptr) a.dres_scale[c] = a.gamma_post != nullptr ? s * a.gamma_post[c] : s;
        if (a.dgamma_post != nullptr) a.dgamma_post[c] = a.res_scale != nullptr ? s * a.res_scale[c] : s;
    } else {
        if (a.res_scale != nullptr) s *= a.res_scale[c];
        if (a.gamma_post != nullptr) s *= a.gamma_post[c];
        const int64_t at = static_cast<int64_t>(job - 2) * a.D + c;
        if (D::BYTES == 4) static_cast<float*>(a.dgate)[at] = s;
        else static_cast<__nv_bfloat16*>(a.dgate)[at] = __float2bfloat16_rn(s);
    }
}


// `shared`: the gradient of a gate shared by several rows is wanted.
NormCut norm_cut(int64_t M, int64_t gate_rows, int D, int tpr, bool shared) {
    NormCut c{};
    const int rows = cta(tpr) / tpr;
    const int64_t ctas_most = static_cast<int64_t>(SMS) * (tpr > 256 ? 1 : BACK_CTAS);
    c.rows = shared && gate_rows < M ? gate_rows : M;
    const int64_t parts = (M + c.rows - 1) / c.rows, want = ctas_most * rows;
    c.spans = (want + parts - 1) / parts;
    if (c.spans > c.rows) c.spans = c.rows;
    c.span = (c.rows + c.spans - 1) / c.spans;
    c.spans = (c.rows + c.span - 1) / c.span;
    c.items = parts * c.spans;
    const int64_t ctas = (c.items + rows - 1) / rows;
    c.grid = static_cast<unsigned>(ctas < ctas_most ? ctas : ctas_most);
    c.groups = static_cast<int>(c.grid) * rows;
    c.gate_at = static_cast<size_t>(2) * c.groups * D;
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

// Rows on their way, of N arrays: four, or what shared memory holds.
template <class D, int TPR, int VE, int N>
constexpr size_t stage_bytes() { return static_cast<size_t>(cta(TPR)) * VE * D::BYTES * N; }
template <class D, int TPR, int VE, int N>
constexpr int stages(int ctas) {
    const size_t most = 200 * 1024 / (TPR > 256 ? 1 : ctas) / stage_bytes<D, TPR, VE, N>();
    return most > 4 ? 4 : static_cast<int>(most);
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
        constexpr int rows = cta(T.value) / T.value;
        const int64_t most = static_cast<int64_t>(SMS) * (T.value > 256 ? 1 : FORE_CTAS) * rows;
        const int64_t span = (a.M + most - 1) / most, groups = (a.M + span - 1) / span;
        constexpr int S = stages<D, T.value, V.value, 2>(FORE_CTAS);
        constexpr size_t smem = S * stage_bytes<D, T.value, V.value, 2>();
        static std::atomic<unsigned long long> seen;
        const cudaError_t e = allow_smem(k_block_norm<D, T.value, V.value, S>, smem, seen);
        if (e != cudaSuccess) return e;
        k_block_norm<D, T.value, V.value, S><<<static_cast<unsigned>((groups + rows - 1) / rows), cta(T.value), smem, stream>>>(a, span);
        return cudaGetLastError();
    });
}
template <class D>
cudaError_t backward(const RowPlan& p, const BlockNorm& a, cudaStream_t stream) {
    const bool shared = a.dgate != nullptr && a.gate_rows > 1;
    const NormCut cut = norm_cut(a.M, a.gate_rows, a.D, p.tpr, shared);
    cudaError_t e = with_plan(p, [&](auto T, auto V) {
        constexpr int S = stages<D, T.value, V.value, 4>(BACK_CTAS);
        constexpr size_t smem = S * stage_bytes<D, T.value, V.value, 4>();
        static std::atomic<unsigned long long> seen;
        const cudaError_t e = allow_smem(k_block_norm_backward<D, T.value, V.value, S>, smem, seen);
        if (e != cudaSuccess) return e;
        k_block_norm_backward<D, T.value, V.value, S><<<cut.grid, cta(T.value), smem, stream>>>(a, cut);
        return cudaGetLastError();
    });
    if (e != cudaSuccess || (a.dgamma_pre == nullptr && a.dgamma_post == nullptr && a.dres_scale == nullptr && !(shared && cut.spans > 1))) return e;
    const int64_t jobs = 2 + (shared && cut.spans > 1 ? cut.items / cut.spans : 0);
    k_block_norm_join<D><<<static_cast<unsigned>(jobs * ((a.D + JC - 1) / JC)), JC * JR, 0, stream>>>(a, cut);
    return cudaGetLastError();
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
    const size_t one = norm_cut(M, gate_rows, D, tpr, false).total, each = norm_cut(M, gate_rows, D, tpr, gate_rows > 1).total;
    return (one > each ? one : each) * 4;
}
cudaError_t launch_block_norm_backward(int dtype, const BlockNorm& a, cudaStream_t stream) {
    const RowPlan p = row_plan(a.D);
    return dtype == SDM_F32 ? backward<F32>(p, a, stream) : backward<BF16>(p, a, stream);
}

}  // namespace sdm
