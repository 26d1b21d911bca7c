// Norms after and before a block, with its gate, residual scale and residual, in one pass over the rows:
//   u = gamma_post y / rms(y),  h = x + res_scale gate u,  z = gamma_pre h / rms(h),  rms(a)^2 = mean a^2 + eps,
// and their gradients.  With n = h / rms(h) of the stored h, n' = y / rms(y) and c = res_scale gamma_post:
//   dx = dh + (dn - n mean(dn n)) / rms(h),  dn = gamma_pre dz;
//   dy = (dn' - n' mean(dn' n')) / rms(y),   dn' = dx gate c, whose mean follows from sums that need neither norm, so that
//   a row takes one reduction;
//   dgamma_pre = sum dz n;  with q = dx n':  dgate = c sum q over the gate's rows,
//   G = sum gate q over all:  dres_scale = gamma_post G,  dgamma_post = res_scale G.
// So two column sums are all that the gradients of four vectors take.
//
// Bound by memory: everything is read once and written once, next rows on their way in shared memory (without: 126 and 213
// us for rows of 2,048), the vectors in registers.  32,768 rows of 2,048 in bf16: forward 99 us, 5.4 TB/s, 0.80 of the copy bandwidth;
// backward 151 us, 5.3 TB/s, 0.78, where the warps' issue slots are two thirds taken and the column sums' registers leave
// two CTAs an SM.  One row: 6 and 11 us, one launch and two.  Sums over a row: TPR threads a row, butterflies
// within a warp, then the warps' shares through shared memory.
#include "dla_internal.h"
#include "sdm_common.cuh"

#include <type_traits>

namespace sdm {

namespace {

// Threads of a CTA: one row or, where a row takes 128 or fewer, several.
__host__ __device__ constexpr int cta(int tpr) { return tpr < 256 ? 256 / tpr * tpr : tpr; }

template <class D>
__device__ __forceinline__ uint4 load16(const void* base, int64_t at) {
    return __ldcs(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(base) + at));
}
template <class D>
__device__ __forceinline__ void store16(void* base, int64_t at, const uint4& u) {
    *reinterpret_cast<uint4*>(static_cast<typename D::T*>(base) + at) = u;
}
// Values in pairs: the packed units take two at once.
template <int P>
__device__ __forceinline__ void put_pairs(float* to, const float2 (&f)[P]) {
#pragma unroll
    for (int p = 0; p < P; p += 2) *reinterpret_cast<float4*>(to + 2 * p) = make_float4(f[p].x, f[p].y, f[p + 1].x, f[p + 1].y);
}
__device__ __forceinline__ float2 two(float x) { return make_float2(x, x); }
// The values at column c of a vector, or ones where it is missing.
template <int P>
__device__ __forceinline__ void ones_or(const float* v, int c, float2 (&f)[P]) {
#pragma unroll
    for (int p = 0; p < P; p += 2) {
        const float4 a = v != nullptr ? __ldg(reinterpret_cast<const float4*>(v + c + 2 * p)) : make_float4(1.f, 1.f, 1.f, 1.f);
        f[p] = make_float2(a.x, a.y);
        f[p + 1] = make_float2(a.z, a.w);
    }
}
template <int P>
__device__ __forceinline__ void product(const float* v, const float* w, int c, float2 (&f)[P]) {
    float2 g[P];
    ones_or<P>(v, c, f);
    ones_or<P>(w, c, g);
#pragma unroll
    for (int p = 0; p < P; ++p) f[p] = __fmul2_rn(f[p], g[p]);
}

// Sums of up to eight values over the TPR threads of a row, the same in all of them; other rows' threads are not waited
// for.  The lanes first halve the values they hold at every step (9 shuffles for eight values, 5 for one), then add up one each.
// `sh`: two sets of the warps' shares, used in turn, so that a sum's shares do not meet the readers of the one before.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float (*sh)[16][8], int& turn) {
    const int lane = threadIdx.x & 31;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < N ? s[i] : 0.f;
    if (N == 1) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        s[0] = v[0];
    } else {
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
        }
    }
    if (TPR == 32) return;
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

// CTAs on an SM: of 256 threads three with 80 registers each (four are no faster: 99 to 100 us for rows of 2,048, three 99), and
// for the gradients two with 128.
constexpr int SMS = 152;
__host__ __device__ constexpr int fore_ctas(int tpr) { return tpr > 256 ? 1 : 768 / cta(tpr); }
__host__ __device__ constexpr int back_ctas(int tpr) { return tpr > 256 ? 1 : 512 / cta(tpr); }

// Threads a row, values a thread in pieces of 16 bytes, rows of a CTA at once.
template <class D, int TPR, int VE>
struct Row {
    static constexpr int E = D::E, P = E / 2, V = VE / E, ROWS = cta(TPR) / TPR;
    // The vectors' values of a thread stay in registers (8,192 rows of 8,192: 96 and 169 us, read again for each row 133 and 280).
    // With 32 of each there are not enough registers, and they are read again; the gradients' sums spill all the same.
    static constexpr bool KEEP = VE <= 16;
};
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
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) copy(s, src);
        }
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

// A group of TPR threads takes `span` rows one after the other.  ROWGATE: every row has its gate, which comes with the row.
template <class D, int TPR, int VE, int S, bool ROWGATE>
__global__ void __launch_bounds__(cta(TPR), fore_ctas(TPR)) k_block_norm(const BlockNorm a, const int64_t span) {
    extern __shared__ __align__(16) unsigned char ring[];
    using R = Row<D, TPR, VE>;
    constexpr int E = R::E, P = R::P, V = R::V;
    __shared__ __align__(16) float sh[2][16][8];
    int turn = 0;
    const int lane = threadIdx.x % TPR;
    const float inv = 1.f / static_cast<float>(a.D);
    const bool post = a.gamma_post != nullptr, has_y = a.y != nullptr, pre = a.z != nullptr;
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * R::ROWS + threadIdx.x / TPR) * span;
    const int64_t last = first + span < a.M ? first + span : a.M;
    if (first >= last) return;
    uint4 gu[V];
    constexpr int N = ROWGATE ? 3 : 2;
    const void* from[N];
    from[0] = a.x;
    from[1] = a.y;
    if (ROWGATE) from[N - 1] = a.gate;
    const void* const (&src)[N] = from;
    Ahead<D, TPR, VE, N, S> rows(ring, first, last, a.D);
    rows.start(src);
    auto gate = [&](int64_t g) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            gu[i] = c < a.D ? __ldg(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(a.gate) + g * a.D + c)) : make_uint4(0, 0, 0, 0);
        }
    };
    const bool shared = !ROWGATE && a.gate != nullptr;
    int64_t g = shared ? first / a.gate_rows : 0, until = shared ? (g + 1) * a.gate_rows : last;
    if (shared) gate(g);
    float2 ck[R::KEEP ? V : 1][P], pk[R::KEEP ? V : 1][P];
    if (R::KEEP) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            if (c < a.D) {
                product<P>(a.res_scale, a.gamma_post, c, ck[i]);
                ones_or<P>(a.gamma_pre, c, pk[i]);
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
            if (ROWGATE) gu[i] = rows.get(src, m, N - 1, i);
        }
        rows.advance(src);
        if (m == until) {
            gate(++g);
            until += a.gate_rows;
        }
        float r = 1.f;
        if (post) {
            float2 q = two(0.f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float2 y[4];
                unpack16x2<D>(yu[i], y);
#pragma unroll
                for (int p = 0; p < P; ++p) q = __ffma2_rn(y[p], y[p], q);
            }
            float s[1] = {q.x + q.y};
            row_sum<TPR>(s, sh, turn);
            r = rsqrtf(fmaf(s[0], inv, a.eps));
        }
        if (has_y) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                float2 x[4], y[4], k[P];
                unpack16x2<D>(xu[i], x);
                unpack16x2<D>(yu[i], y);
                if (!R::KEEP) product<P>(a.res_scale, a.gamma_post, c, k);
                if (ROWGATE || shared) {
                    float2 ga[4];
                    unpack16x2<D>(gu[i], ga);
#pragma unroll
                    for (int p = 0; p < P; ++p) y[p] = __fmul2_rn(y[p], ga[p]);
                }
#pragma unroll
                for (int p = 0; p < P; ++p) x[p] = __ffma2_rn(__fmul2_rn(y[p], two(r)), R::KEEP ? ck[i][p] : k[p], x[p]);
                xu[i] = pack16x2<D>(x);
                store16<D>(a.h, m * a.D + c, xu[i]);
            }
        }
        if (!pre) continue;
        float2 q = two(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {                        // of what is stored
            float2 x[4];
            unpack16x2<D>(xu[i], x);
#pragma unroll
            for (int p = 0; p < P; ++p) q = __ffma2_rn(x[p], x[p], q);
        }
        float s[1] = {q.x + q.y};
        row_sum<TPR>(s, sh, turn);
        r = rsqrtf(fmaf(s[0], inv, a.eps));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            if (c >= a.D) continue;
            float2 x[4], k[P];
            unpack16x2<D>(xu[i], x);
            if (!R::KEEP) ones_or<P>(a.gamma_pre, c, k);
#pragma unroll
            for (int p = 0; p < P; ++p) x[p] = __fmul2_rn(__fmul2_rn(x[p], two(r)), R::KEEP ? pk[i][p] : k[p]);
            store16<D>(a.z, m * a.D + c, pack16x2<D>(x));
        }
    }
}

// The gradients.  A group of TPR threads takes `span` rows one after the other.  Column sums stay in registers: dz n's over
// all of them, q's over the rows of one gate (times the gate it is those rows' share of G, which the group adds up in
// `ws`), or, where every row has its gate (ROWGATE), G's own.  A gate whose rows one group has is done with there; a
// gate of several groups has a share from each, the group's first or second (a gate that starts within its rows).  Shares are
// joined in order.
struct NormCut {
    int64_t span;
    unsigned grid;
    int groups;                  // of all CTAs
    size_t gate_at, total;       // floats of `ws`: [2][groups][D], then [groups][2][D] where a gate may have several groups
};

template <class D, int TPR, int VE, int S, bool ROWGATE>
__global__ void __launch_bounds__(cta(TPR), back_ctas(TPR)) k_block_norm_backward(const BlockNorm a, const NormCut cut) {
    extern __shared__ __align__(16) unsigned char ring[];
    using R = Row<D, TPR, VE>;
    constexpr int E = R::E, P = R::P, V = R::V;
    __shared__ __align__(16) float sh[2][16][8];
    int turn = 0;
    const int lane = threadIdx.x % TPR, group = blockIdx.x * R::ROWS + threadIdx.x / TPR;
    const float inv = 1.f / static_cast<float>(a.D);
    const bool post = a.gamma_post != nullptr, pre = a.dz != nullptr, has_y = a.y != nullptr, has_gate = a.gate != nullptr;
    float2 sp[V][P], sq[V][P];                               // sums of dz n and of q
    float2 ck[R::KEEP ? V : 1][P], pk[R::KEEP ? V : 1][P];   // c (times the gate, unless that is the row's) and gamma_pre
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (lane + i * TPR) * E;
#pragma unroll
        for (int p = 0; p < P; ++p) sp[i][p] = sq[i][p] = two(0.f);
        if (R::KEEP && c < a.D) {
            product<P>(a.res_scale, a.gamma_post, c, ck[i]);
            ones_or<P>(a.gamma_pre, c, pk[i]);
        }
    }
    constexpr int N = ROWGATE ? 5 : 4;
    const void* src[N];
    src[0] = pre ? a.h : nullptr;
    src[1] = a.dz;
    src[2] = a.y;
    src[3] = a.dh;
    if (ROWGATE) src[N - 1] = a.gate;
    const void* const (&from)[N] = src;
    auto gate_at = [&](int64_t g, int c, float2 (&f)[4]) {
        unpack16x2<D>(__ldg(reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(a.gate) + g * a.D + c)), f);
    };
    bool added = false;                                      // a share of G is in `ws`
    const int64_t first = group * cut.span;
    const int64_t last = first + cut.span < a.M ? first + cut.span : a.M;
    int64_t g = 0, until = !ROWGATE && has_gate ? first : last;      // the gate's row at hand, and its end
    Ahead<D, TPR, VE, N, S> rows(ring, first, last, a.D);
    rows.start(from);
    for (int64_t m = first; m < last; ++m) {
        uint4 hu[V], yu[V], zu[V], du[V], gu[V];
        rows.wait();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            hu[i] = rows.get(from, m, 0, i);
            zu[i] = rows.get(from, m, 1, i);
            yu[i] = rows.get(from, m, 2, i);
            du[i] = rows.get(from, m, 3, i);
            if (ROWGATE) gu[i] = rows.get(from, m, N - 1, i);
        }
        rows.advance(from);
        if (m == until) {
            g = m / a.gate_rows;
            until = (g + 1) * a.gate_rows;
            if (R::KEEP) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (lane + i * TPR) * E;
                    if (c >= a.D) continue;
                    float2 ga[4];
                    gate_at(g, c, ga);
                    product<P>(a.res_scale, a.gamma_post, c, ck[i]);
#pragma unroll
                    for (int p = 0; p < P; ++p) ck[i][p] = __fmul2_rn(ck[i][p], ga[p]);
                }
            }
        }
        auto gate_c = [&](int c, float2 (&k)[P]) {       // where it is not kept
            product<P>(a.res_scale, a.gamma_post, c, k);
            if (ROWGATE || !has_gate) return;
            float2 ga[4];
            gate_at(g, c, ga);
#pragma unroll
            for (int p = 0; p < P; ++p) k[p] = __fmul2_rn(k[p], ga[p]);
        };
        // sums of h^2, dn h, y^2 and, with b = gate c y, of b dh, b dn and b h
        float2 t[6];
#pragma unroll
        for (int j = 0; j < 6; ++j) t[j] = two(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            if (c >= a.D) continue;
            float2 h[4], z[4], y[4], d[4], k[P], kc[P];
            unpack16x2<D>(hu[i], h);
            unpack16x2<D>(zu[i], z);
            unpack16x2<D>(yu[i], y);
            unpack16x2<D>(du[i], d);
            if (!R::KEEP) ones_or<P>(a.gamma_pre, c, k);
            if (!R::KEEP) gate_c(c, kc);
            if (ROWGATE) {
                float2 ga[4];
                unpack16x2<D>(gu[i], ga);
#pragma unroll
                for (int p = 0; p < P; ++p) kc[p] = __fmul2_rn(ga[p], R::KEEP ? ck[i][p] : kc[p]);
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const float2 n = __fmul2_rn(z[p], R::KEEP ? pk[i][p] : k[p]), b = __fmul2_rn(y[p], R::KEEP && !ROWGATE ? ck[i][p] : kc[p]);
                t[0] = __ffma2_rn(h[p], h[p], t[0]);
                t[1] = __ffma2_rn(n, h[p], t[1]);
                t[2] = __ffma2_rn(y[p], y[p], t[2]);
                t[3] = __ffma2_rn(b, d[p], t[3]);
                t[4] = __ffma2_rn(b, n, t[4]);
                t[5] = __ffma2_rn(b, h[p], t[5]);
            }
        }
        float s[6];
#pragma unroll
        for (int j = 0; j < 6; ++j) s[j] = t[j].x + t[j].y;
        if (pre || post) row_sum<TPR>(s, sh, turn);
        const float rh = pre ? rsqrtf(fmaf(s[0], inv, a.eps)) : 0.f, ch = s[1] * rh * rh * inv;      // mean(dn n) rh = ch rh; n = h rh
        const float ry = post ? rsqrtf(fmaf(s[2], inv, a.eps)) : 1.f;
        // mean(dn' n') = ry mean(b dx), dx = dh + rh (dn - h ch)
        const float mean = post ? ry * inv * (pre ? s[3] + rh * (s[4] - ch * s[5]) : s[3]) : 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (lane + i * TPR) * E;
            if (c >= a.D) continue;
            float2 dx[4], k[P];
            unpack16x2<D>(du[i], dx);
            if (pre) {
                float2 h[4], z[4];
                unpack16x2<D>(hu[i], h);
                unpack16x2<D>(zu[i], z);
                if (!R::KEEP) ones_or<P>(a.gamma_pre, c, k);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    sp[i][p] = __ffma2_rn(z[p], __fmul2_rn(h[p], two(rh)), sp[i][p]);
                    dx[p] = __ffma2_rn(two(rh), __ffma2_rn(h[p], two(-ch), __fmul2_rn(z[p], R::KEEP ? pk[i][p] : k[p])), dx[p]);
                }
            }
            store16<D>(a.dx, m * a.D + c, pack16x2<D>(dx));
            if (!has_y) continue;
            float2 y[4];
            unpack16x2<D>(yu[i], y);
#pragma unroll
            for (int p = 0; p < P; ++p) y[p] = __fmul2_rn(y[p], two(ry));        // n': y itself without a norm
            if (!R::KEEP) gate_c(c, k);
            if (ROWGATE) {
                float2 ga[4], q[4];
                unpack16x2<D>(gu[i], ga);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float2 ce = R::KEEP ? ck[i][p] : k[p];
                    q[p] = __fmul2_rn(dx[p], y[p]);
                    sq[i][p] = __ffma2_rn(ga[p], q[p], sq[i][p]);
                    q[p] = __fmul2_rn(q[p], ce);
                    dx[p] = __fmul2_rn(dx[p], __fmul2_rn(ga[p], ce));
                }
                if (a.dgate != nullptr) store16<D>(a.dgate, m * a.D + c, pack16x2<D>(q));
            } else {
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    sq[i][p] = __ffma2_rn(dx[p], y[p], sq[i][p]);
                    dx[p] = __fmul2_rn(dx[p], R::KEEP ? ck[i][p] : k[p]);
                }
            }
            if (post) {
#pragma unroll
                for (int p = 0; p < P; ++p) dx[p] = __fmul2_rn(two(ry), __ffma2_rn(y[p], two(-mean), dx[p]));
            }
            store16<D>(a.dy, m * a.D + c, pack16x2<D>(dx));
        }
        if (!ROWGATE && has_gate && (m + 1 == last || m + 1 == until)) {         // the gate's share of G, and its own sum
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (lane + i * TPR) * E;
                if (c >= a.D) continue;
                float2 ga[4], k[4], f[P];
                gate_at(g, c, ga);
                float* const at = a.ws + (static_cast<int64_t>(cut.groups) + group) * a.D + c;
#pragma unroll
                for (int p = 0; p < P; ++p) f[p] = __fmul2_rn(ga[p], sq[i][p]);
                if (added) {
#pragma unroll
                    for (int p = 0; p < P; ++p) f[p] = __fadd2_rn(f[p], *reinterpret_cast<const float2*>(at + 2 * p));
                }
                put_pairs<P>(at, f);
                if (a.dgate != nullptr) {
                    const int64_t from_row = g * a.gate_rows, to_row = until < a.M ? until : a.M;
                    if (from_row < first || to_row > last) {
                        put_pairs<P>(a.ws + cut.gate_at + (2 * static_cast<int64_t>(group) + (from_row > first)) * a.D + c, sq[i]);
                    } else {
                        float2 kc[P];
                        product<P>(a.res_scale, a.gamma_post, c, kc);
#pragma unroll
                        for (int p = 0; p < P; ++p) k[p] = __fmul2_rn(sq[i][p], kc[p]);
                        store16<D>(a.dgate, g * a.D + c, pack16x2<D>(k));
                    }
                }
#pragma unroll
                for (int p = 0; p < P; ++p) sq[i][p] = two(0.f);
            }
            added = true;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (lane + i * TPR) * E;
        if (c >= a.D) continue;
        float* const at = a.ws + static_cast<int64_t>(group) * a.D + c;
        put_pairs<P>(at, sp[i]);
        if (!added) put_pairs<P>(at + static_cast<int64_t>(cut.groups) * a.D, sq[i]);
    }
}

// Sums over the shares, in order: JC columns a CTA, JR ranges of groups.  Job 0: dgamma_pre, 1: dres_scale and dgamma_post from
// G, 2 and on: the gates of several groups, a CTA every so many'th.
constexpr int JC = 16, JR = 16, GATE_JOBS = 16;
template <class D>
__global__ void __launch_bounds__(JC * JR) k_block_norm_join(const BlockNorm a, const NormCut cut, const int64_t gates) {
    __shared__ float sum[JR][JC + 1];
    const unsigned cols = static_cast<unsigned>((a.D + JC - 1) / JC), job = blockIdx.x / cols;
    const int x = threadIdx.x % JC, y = threadIdx.x / JC, c = static_cast<int>(blockIdx.x - job * cols) * JC + x;
    auto total = [&](float s) {                              // in the threads of y = 0
        __syncthreads();
        sum[y][x] = s;
        __syncthreads();
        for (int i = 1; i < JR; ++i) s += sum[i][x];
        return s;
    };
    if (job < 2) {
        if (job == 0 ? a.dgamma_pre == nullptr : a.dgamma_post == nullptr && a.dres_scale == nullptr) return;
        const float* p = a.ws + static_cast<int64_t>(job) * cut.groups * a.D + c;
        float s = 0.f;
        if (c < a.D)
#pragma unroll 8
            for (int i = y; i < cut.groups; i += JR) s += __ldcs(p + static_cast<int64_t>(i) * a.D);
        s = total(s);
        if (y != 0 || c >= a.D) return;
        if (job == 0) {
            a.dgamma_pre[c] = s;
            return;
        }
        if (a.dres_scale != nullptr) a.dres_scale[c] = a.gamma_post != nullptr ? s * a.gamma_post[c] : s;
        if (a.dgamma_post != nullptr) a.dgamma_post[c] = a.res_scale != nullptr ? s * a.res_scale[c] : s;
        return;
    }
    // where gates outnumber groups, the gates at the groups' ends are all that may have several
    const bool ends = gates > cut.groups;
    const int64_t jobs = ends ? cut.groups : gates;
    for (int64_t j = job - 2; j < jobs; j += GATE_JOBS) {
        const int64_t last = (j + 1) * cut.span - 1;
        if (ends && last >= a.M) break;
        const int64_t g = ends ? last / a.gate_rows : j, from = g * a.gate_rows, to = from + a.gate_rows < a.M ? from + a.gate_rows : a.M;
        const int64_t g0 = from / cut.span, g1 = (to - 1) / cut.span;
        if (g0 == g1 || (ends && g0 != j)) continue;
        float s = 0.f;
        if (c < a.D)
            for (int64_t i = g0 + y; i <= g1; i += JR) s += __ldcs(a.ws + cut.gate_at + (2 * i + (from > i * cut.span)) * a.D + c);
        s = total(s);
        if (y != 0 || c >= a.D) continue;
        if (a.res_scale != nullptr) s *= a.res_scale[c];
        if (a.gamma_post != nullptr) s *= a.gamma_post[c];
        const int64_t at = g * a.D + c;
        if (D::BYTES == 4) static_cast<float*>(a.dgate)[at] = s;
        else static_cast<__nv_bfloat16*>(a.dgate)[at] = __float2bfloat16_rn(s);
    }
}

// `shared`: the gradient of a gate shared by several rows is wanted.
NormCut norm_cut(int64_t M, int D, int tpr, bool shared) {
    NormCut c{};
    const int rows = cta(tpr) / tpr;
    const int64_t most = static_cast<int64_t>(SMS) * back_ctas(tpr) * rows;
    c.span = (M + most - 1) / most;
    const int64_t groups = (M + c.span - 1) / c.span;
    c.grid = static_cast<unsigned>((groups + rows - 1) / rows);
    c.groups = static_cast<int>(c.grid) * rows;
    c.gate_at = static_cast<size_t>(2) * c.groups * D;
    c.total = c.gate_at + (shared ? static_cast<size_t>(2) * c.groups * D : 0);
    return c;
}

// Threads a row and values a thread: eight values (16 make the registers of the gradients' sums: bf16 rows of 2,048 103 and 204 us forward
// and backward, with eight 99 and 151) in up to 256 threads, as several CTAs of an SM hide each other's waits.  Then it is what
// moves with two 16-byte pieces of an array a thread: 16 bf16 values (rows of 4,096: 102 and 152 us, 512 threads of eight 107 and 173) or
// 512 threads of eight float32 values (98 and 152, 256 of 16 101 and 231).  Then 512 threads of 16 and 32.
// A power of two leaves threads without work where the width is none.  bf16 gradients, 134 MB an array: rows of 768 by 96 threads
// 146 us, by 128 180; 1,280 by 160 154, by 256 204; 1,536 by 192 156, by 256 190; 2,560 by 160 of 16 163, by 256 193.  Forward: 101 and
// 94, 97 and 115, 101 and 101, 99 and 98 (with a gate a row 117 and 112), so there it is 160 threads of eight alone.
// Wider rows leave one CTA of 512 threads an SM, and the gradients of 16 float32 and of 32 values spill (234 and 844 bytes in float32, 338
// in bf16) and have one row on its way or none.  134 MB an array, forward and backward: float32 rows of 4,096 98 and 149 us, 5,120 98 and
// 241, 8,192 95 and 233, 16,384 120 and 355; bf16 rows of 5,120 107 and 210, 6,144 93 and 188, 8,192 96 and 169, 10,240 155 and 387, 16,384 132
// and 338.
struct RowPlan {
    int tpr, ve;
};
RowPlan row_plan(int dtype, int D, bool back) {
    if (dtype == SDM_BF16) {
        for (const RowPlan p : {RowPlan{32, 8}, {64, 8}, {96, 8}, {128, 8}, {160, 8}, {192, 8}, {256, 8}, {160, 16}, {256, 16}})
            if (p.tpr * p.ve >= D && (back || (p.tpr & (p.tpr - 1)) == 0 || (p.tpr == 160 && p.ve == 8))) return p;
    }
    RowPlan p{32, 8};
    while (p.tpr < 256 && p.tpr * p.ve < D) p.tpr *= 2;
    if (p.tpr * p.ve < D) p.tpr = 512;
    while (p.tpr * p.ve < D) p.ve *= 2;
    return p;
}

// Rows on their way, of N arrays: four, or what shared memory holds.
template <class D, int TPR, int VE, int N>
constexpr size_t stage_bytes() { return static_cast<size_t>(cta(TPR)) * VE * D::BYTES * N; }
template <class D, int TPR, int VE, int N>
constexpr int stages(int ctas) {
    const size_t most = 200 * 1024 / ctas / stage_bytes<D, TPR, VE, N>();
    return most > 4 ? 4 : static_cast<int>(most);
}

template <class D, bool BACK, class F>
cudaError_t with_plan(const RowPlan& p, F f) {
#define SDM_ROW(T, V) if (p.tpr == (T) && p.ve == (V)) return f(std::integral_constant<int, T>{}, std::integral_constant<int, V>{});
    if constexpr (D::BYTES == 2) {
        if constexpr (BACK) {
            SDM_ROW(96, 8) SDM_ROW(192, 8) SDM_ROW(160, 16)
        }
        SDM_ROW(160, 8) SDM_ROW(256, 16)
    } else {
        SDM_ROW(512, 8)
    }
    SDM_ROW(32, 8) SDM_ROW(64, 8) SDM_ROW(128, 8) SDM_ROW(256, 8) SDM_ROW(512, 16) SDM_ROW(512, 32)
#undef SDM_ROW
    return cudaErrorInvalidValue;
}

template <class D, bool ROWGATE>
cudaError_t forward(const RowPlan& p, const BlockNorm& a, cudaStream_t stream) {
    return with_plan<D, false>(p, [&](auto T, auto V) {
        constexpr int rows = cta(T.value) / T.value;
        const int64_t most = static_cast<int64_t>(SMS) * fore_ctas(T.value) * rows;
        const int64_t span = (a.M + most - 1) / most, groups = (a.M + span - 1) / span;
        constexpr int N = ROWGATE ? 3 : 2, S = stages<D, T.value, V.value, N>(fore_ctas(T.value));
        constexpr size_t smem = S * stage_bytes<D, T.value, V.value, N>();
        static std::atomic<unsigned long long> seen;
        const cudaError_t e = allow_smem(k_block_norm<D, T.value, V.value, S, ROWGATE>, smem, seen);
        if (e != cudaSuccess) return e;
        k_block_norm<D, T.value, V.value, S, ROWGATE><<<static_cast<unsigned>((groups + rows - 1) / rows), cta(T.value), smem, stream>>>(a, span);
        return cudaGetLastError();
    });
}
template <class D, bool ROWGATE>
cudaError_t backward(const RowPlan& p, const BlockNorm& a, cudaStream_t stream) {
    const bool shared = a.dgate != nullptr && a.gate_rows > 1;
    const NormCut cut = norm_cut(a.M, a.D, p.tpr, shared);
    cudaError_t e = with_plan<D, true>(p, [&](auto T, auto V) {
        constexpr int S = stages<D, T.value, V.value, ROWGATE ? 5 : 4>(back_ctas(T.value));
        constexpr size_t smem = S * stage_bytes<D, T.value, V.value, ROWGATE ? 5 : 4>();
        static std::atomic<unsigned long long> seen;
        const cudaError_t e = allow_smem(k_block_norm_backward<D, T.value, V.value, S, ROWGATE>, smem, seen);
        if (e != cudaSuccess) return e;
        k_block_norm_backward<D, T.value, V.value, S, ROWGATE><<<cut.grid, cta(T.value), smem, stream>>>(a, cut);
        return cudaGetLastError();
    });
    if (e != cudaSuccess || (a.dgamma_pre == nullptr && a.dgamma_post == nullptr && a.dres_scale == nullptr && !shared)) return e;
    const int64_t gates = shared ? (a.M + a.gate_rows - 1) / a.gate_rows : 0, gate_jobs = gates < GATE_JOBS ? gates : GATE_JOBS;
    k_block_norm_join<D><<<static_cast<unsigned>((2 + gate_jobs) * ((a.D + JC - 1) / JC)), JC * JR, 0, stream>>>(a, cut, gates);
    return cudaGetLastError();
}

}  // namespace

bool block_norm_supported(int D) { return D <= 512 * 32; }
cudaError_t launch_block_norm(int dtype, const BlockNorm& a, cudaStream_t stream) {
    const RowPlan p = row_plan(dtype, a.D, false);
    if (a.gate != nullptr && a.gate_rows == 1) return dtype == SDM_F32 ? forward<F32, true>(p, a, stream) : forward<BF16, true>(p, a, stream);
    return dtype == SDM_F32 ? forward<F32, false>(p, a, stream) : forward<BF16, false>(p, a, stream);
}
size_t block_norm_backward_bytes(int dtype, int64_t M, int64_t gate_rows, int D) {
    if (M == 0) return 0;
    return norm_cut(M, D, row_plan(dtype, D, true).tpr, gate_rows > 1).total * 4;
}
cudaError_t launch_block_norm_backward(int dtype, const BlockNorm& a, cudaStream_t stream) {
    const RowPlan p = row_plan(dtype, a.D, true);
    if (a.gate != nullptr && a.gate_rows == 1) return dtype == SDM_F32 ? backward<F32, true>(p, a, stream) : backward<BF16, true>(p, a, stream);
    return dtype == SDM_F32 ? backward<F32, false>(p, a, stream) : backward<BF16, false>(p, a, stream);
}

}  // namespace sdm
