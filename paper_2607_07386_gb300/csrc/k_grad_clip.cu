// The global norm of many gradients, and clipping by it:
//   norm = sqrt(sum over all tensors of g^2),  out = g min(1, max_norm / norm).
//
// Bound by memory: one pass reads everything for the norm, the second reads it again and writes.  Both cut the list's blocks
// of 32 KB into one range a CTA, and the second walks every range backwards, so that what the first read last is still in L2.
// The loads of a block are on their way while the one before is worked on.
//
// 1.15 GB: the norm in 181 us (6.4 TB/s), with the scaling 549 (0.93 of the copy bandwidth for three passes).
//
// The list goes to the kernels in their parameters: nothing is copied to the device first, and a captured launch holds its
// list.  A CTA's sums go to the workspace and are joined in order (by every CTA of the second pass for itself), so the
// norm is the same on every call.
//
// Squares of float32 values run out of float32's range at 2^64 and 2^-63, long before the values do, so three sums are kept:
// of x^2, (2^-80 x)^2 and (2^80 x)^2.  The first counts unless it overflowed or is so small that squares were lost.  Each is a
// float32 sum over the 32 or 64 values of a thread in a block, then compensated over the blocks, then in 64 bits.
#include "dla_internal.h"
#include "sdm_common.cuh"

namespace sdm {

namespace {

constexpr int GT = 256, PIECES = 8;              // threads; pieces of 16 bytes of the gradient a thread
constexpr int64_t BLOCK = GT * PIECES * 16;      // bytes of the gradient a block
constexpr int CTAS = 152 * 2;                    // of 256 threads of up to 128 registers, a launch
// Tensors a launch.  A long table takes longer to launch (3 MB in 28 tensors: 13.0 us, in the short one 12.7), a list in many
// launches longer still (0.8 GB in 96 tensors: 408 us in short tables, 379 in a long one).
constexpr int FEW = 64, MANY = 960;

struct Entry {
    const void* src;
    void* dst;
    int64_t n;
    int first;                                   // the tensor's first block of this launch
    int kind;                                    // bit 0: src is bf16; bit 1: dst is bf16; bit 2: one by one (addresses that do not match)
};
template <int N>
struct GradTable {
    int count, blocks, per;                      // tensors, their blocks, blocks a CTA
    Entry e[N];
};
static_assert(sizeof(GradTable<MANY>) <= 32000, "kernel parameters");

// The tensor of a block.
template <int N>
__device__ __forceinline__ int find(const GradTable<N>& t, int block) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.e[mid].first <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}
constexpr float UP = 1208925819614629174706176.f, DOWN = 1.f / UP;      // 2^80

__device__ __forceinline__ void add_squares(float2 x, float2 (&s)[3]) {
    const float2 d = __fmul2_rn(x, make_float2(DOWN, DOWN)), u = __fmul2_rn(x, make_float2(UP, UP));
    s[0] = __ffma2_rn(x, x, s[0]);
    s[1] = __ffma2_rn(d, d, s[1]);
    s[2] = __ffma2_rn(u, u, s[2]);
}

// Elements of a tensor before its first 16-byte boundary (all of them are whole elements away from it).
template <class D> __device__ __forceinline__ int head_of(const void* p, int64_t n) {
    const int h = static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / D::BYTES;
    return h < n ? h : static_cast<int>(n);
}

// Where the pieces of a block lie.
struct Span {
    const uint4* at;                             // this thread's first
    int64_t left;                                // pieces from there to the tensor's end
};
template <class D>
__device__ __forceinline__ Span span_of(const Entry& e, int block, int& head) {
    head = head_of<D>(e.src, e.n);
    const int64_t first = static_cast<int64_t>(block - e.first) * (GT * PIECES) + threadIdx.x;
    return Span{reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(e.src) + head) + first, (e.n - head) / D::E - first};
}
__device__ __forceinline__ void load_block(const Entry& e, int block, uint4 (&u)[PIECES]) {
    int head;
    const Span p = e.kind & 1 ? span_of<BF16>(e, block, head) : span_of<F32>(e, block, head);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) u[i] = i * GT < p.left ? __ldg(p.at + i * GT) : make_uint4(0, 0, 0, 0);
}
template <class D>
__device__ __forceinline__ void squares(const Entry& e, int block, const uint4 (&u)[PIECES], float2 (&s)[3]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        float2 f[4];
        unpack16x2<D>(u[i], f);
#pragma unroll
        for (int j = 0; j < D::E / 2; ++j) add_squares(f[j], s);
    }
    if (block == e.first) {                      // what lies before and behind the pieces
        const int head = head_of<D>(e.src, e.n);
        const int64_t tail = head + (e.n - head) / D::E * D::E;
        if (threadIdx.x < head) add_squares(make_float2(load_elem<D>(e.src, threadIdx.x), 0.f), s);
        if (tail + threadIdx.x < e.n) add_squares(make_float2(load_elem<D>(e.src, tail + threadIdx.x), 0.f), s);
    }
}

template <int N>
__global__ void __launch_bounds__(GT, 2) k_grad_squares(const __grid_constant__ GradTable<N> t, double* __restrict__ part) {
    __shared__ double sh[GT / 32][3];
    const int b0 = blockIdx.x * t.per, b1 = min(b0 + t.per, t.blocks);
    float hi[3] = {0.f, 0.f, 0.f}, lo[3] = {0.f, 0.f, 0.f};
    int at = find(t, b0);
    uint4 next[PIECES];
    load_block(t.e[at], b0, next);
    for (int b = b0; b < b1; ++b) {
        const Entry& e = t.e[at];
        uint4 u[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) u[i] = next[i];
        if (b + 1 < b1) {
            while (at + 1 < t.count && t.e[at + 1].first <= b + 1) ++at;
            load_block(t.e[at], b + 1, next);
        }
        float2 s2[3] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        if (e.kind & 1) squares<BF16>(e, b, u, s2);
        else squares<F32>(e, b, u, s2);
#pragma unroll
        for (int i = 0; i < 3; ++i) {                        // a block's sum to the blocks', with what the addition leaves
            const float x = s2[i].x + s2[i].y, sum = hi[i] + x, back = sum - hi[i];
            lo[i] += (hi[i] - (sum - back)) + (x - back);
            hi[i] = sum;
        }
    }
    double s[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        // where the sum is infinite, what was left is not a number
        s[i] = fabsf(hi[i]) <= 3.402823466e+38f ? static_cast<double>(hi[i]) + static_cast<double>(lo[i]) : static_cast<double>(hi[i]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    }
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) {
        sh[warp][0] = s[0];
        sh[warp][1] = s[1];
        sh[warp][2] = s[2];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        double x = 0;
        for (int w = 0; w < GT / 32; ++w) x += sh[w][threadIdx.x];
        part[static_cast<int64_t>(blockIdx.x) * 3 + threadIdx.x] = x;
    }
}

// The norm and the factor from the shares, in 64 bits and in order; in every thread of the CTA.
__device__ __forceinline__ float2 norm_of(const double* __restrict__ part, int shares, float max_norm) {
    __shared__ double sh[GT / 32][3];
    double s[3] = {0, 0, 0};
    for (int i = threadIdx.x; i < shares; i += GT)
#pragma unroll
        for (int j = 0; j < 3; ++j) s[j] += __ldg(part + i * 3 + j);
#pragma unroll
    for (int j = 0; j < 3; ++j)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
    if ((threadIdx.x & 31) == 0)
        for (int j = 0; j < 3; ++j) sh[threadIdx.x >> 5][j] = s[j];
    __syncthreads();
    for (int j = 0; j < 3; ++j) {
        s[j] = 0;
        for (int w = 0; w < GT / 32; ++w) s[j] += sh[w][j];
    }
    const double big = 3.4e38, small = 1e-20;    // below, squares of 2^-63 and less may have counted
    double norm = s[0] <= big && s[0] >= small ? sqrt(s[0]) : s[0] < small ? sqrt(s[2]) * static_cast<double>(DOWN) : sqrt(s[1]) * static_cast<double>(UP);
    if (s[0] != s[0]) norm = s[0];
    const float f = static_cast<float>(norm);
    return make_float2(f, !(fabsf(f) <= 3.402823466e+38f) ? __int_as_float(0x7fffffff) : norm > max_norm ? static_cast<float>(max_norm / norm) : 1.f);
}
__global__ void __launch_bounds__(GT) k_grad_norm(const double* __restrict__ part, int shares, float max_norm, float* __restrict__ stats) {
    const float2 f = norm_of(part, shares, max_norm);
    if (threadIdx.x < 2) stats[threadIdx.x] = threadIdx.x == 0 ? f.x : f.y;
}

template <class S, class O>
__device__ __forceinline__ void put_elem(const void* src, void* dst, int64_t i, float f) {
    if (S::BYTES == O::BYTES && f == 1.f) {      // a copy, bit for bit
        static_cast<typename O::T*>(dst)[i] = static_cast<const typename O::T*>(src)[i];
        return;
    }
    const float x = load_elem<S>(src, i) * f;
    if (O::BYTES == 4) static_cast<float*>(dst)[i] = x;
    else static_cast<__nv_bfloat16*>(dst)[i] = __float2bfloat16_rn(x);
}
// E values of S at once to O.
template <class S, class O> __device__ __forceinline__ void put_piece(void* dst, int64_t i, const float* f) {
    if constexpr (S::E == O::E) {
        *reinterpret_cast<uint4*>(static_cast<typename O::T*>(dst) + i) = pack16<O>(f);
    } else if constexpr (O::BYTES == 4) {        // eight bf16 to two pieces of float32
        *reinterpret_cast<uint4*>(static_cast<float*>(dst) + i) = pack16<F32>(f);
        *reinterpret_cast<uint4*>(static_cast<float*>(dst) + i + 4) = pack16<F32>(f + 4);
    } else {                                     // four float32 to half a piece of bf16
        float g[8] = {f[0], f[1], f[2], f[3], 0.f, 0.f, 0.f, 0.f};
        const uint4 u = pack16<BF16>(g);
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(dst) + i) = make_uint2(u.x, u.y);
    }
}
template <class S, class O>
__device__ __forceinline__ void scale(const Entry& e, int block, const uint4 (&u)[PIECES], float f) {
    if (e.kind & 4) {
        constexpr int64_t per = GT * PIECES * S::E;
        const int64_t first = static_cast<int64_t>(block - e.first) * per, last = first + per < e.n ? first + per : e.n;
        for (int64_t i = first + threadIdx.x; i < last; i += GT) put_elem<S, O>(e.src, e.dst, i, f);
        return;
    }
    int head;
    const Span p = span_of<S>(e, block, head);
    const int64_t first = static_cast<int64_t>(block - e.first) * (GT * PIECES) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        if (i * GT >= p.left) break;
        const int64_t to = head + (first + i * GT) * S::E;
        if (S::BYTES == O::BYTES && f == 1.f) {
            *reinterpret_cast<uint4*>(static_cast<typename O::T*>(e.dst) + to) = u[i];
            continue;
        }
        float x[8];
        unpack16<S>(u[i], x);
#pragma unroll
        for (int j = 0; j < S::E; ++j) x[j] *= f;
        put_piece<S, O>(e.dst, to, x);
    }
    if (block == e.first) {
        const int64_t tail = head + (e.n - head) / S::E * S::E;
        if (threadIdx.x < head) put_elem<S, O>(e.src, e.dst, threadIdx.x, f);
        if (tail + threadIdx.x < e.n) put_elem<S, O>(e.src, e.dst, tail + threadIdx.x, f);
    }
}

template <int N>
__global__ void __launch_bounds__(GT, 2) k_grad_scale(const __grid_constant__ GradTable<N> t, const double* __restrict__ part, int shares, float max_norm,
                                                      float* __restrict__ stats) {
    const int b0 = blockIdx.x * t.per, b1 = min(b0 + t.per, t.blocks);
    int at = find(t, b1 - 1);
    uint4 next[PIECES];
    load_block(t.e[at], b1 - 1, next);           // on its way while the shares are joined
    const float2 nf = norm_of(part, shares, max_norm);
    if (stats != nullptr && blockIdx.x == 0 && threadIdx.x < 2) stats[threadIdx.x] = threadIdx.x == 0 ? nf.x : nf.y;
    const float f = nf.y == nf.y ? nf.y : 1.f;   // the norm is not finite: the gradients stay as they are
    for (int b = b1 - 1; b >= b0; --b) {
        const Entry& e = t.e[at];
        uint4 u[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) u[i] = next[i];
        if (b > b0) {
            while (t.e[at].first > b - 1) --at;
            if (f != 1.f || t.e[at].src != t.e[at].dst) load_block(t.e[at], b - 1, next);
        }
        if (f == 1.f && e.src == e.dst) continue;
        switch (e.kind & 3) {
            case 0: scale<F32, F32>(e, b, u, f); break;
            case 1: scale<BF16, F32>(e, b, u, f); break;
            case 2: scale<F32, BF16>(e, b, u, f); break;
            default: scale<BF16, BF16>(e, b, u, f); break;
        }
    }
}

int64_t blocks_of(const sdm_grad_tensor& t) {
    const int64_t bytes = t.n * (t.dtype == SDM_F32 ? 4 : 2);
    return (bytes + BLOCK - 1) / BLOCK;
}
// The next launch's table; `i` goes past what it took.  All blocks fit an int: a list has up to 2^40 values in 2^24 tensors, 2^27 + 2^24 blocks.
template <int N>
void fill(GradTable<N>& t, int64_t n, const sdm_grad_tensor* list, int64_t& i) {
    t.count = 0;
    int64_t blocks = 0;
    for (; i < n && t.count < N; ++i) {
        const sdm_grad_tensor& g = list[i];
        const int64_t b = blocks_of(g);
        if (b == 0) continue;
        const bool half = g.dtype == SDM_BF16, out_half = g.out_dtype == SDM_BF16;
        // the pieces of src begin on 16 bytes; those of dst must begin on their own size
        const uintptr_t s = reinterpret_cast<uintptr_t>(g.grad), d = reinterpret_cast<uintptr_t>(g.out);
        const uintptr_t head = ((16 - s % 16) % 16) / (half ? 2 : 4) * (out_half ? 2 : 4);
        const uintptr_t need = !half && out_half ? 8 : 16;
        t.e[t.count++] = Entry{g.grad, g.out, g.n, static_cast<int>(blocks), (half ? 1 : 0) | (out_half ? 2 : 0) | ((d + head) % need != 0 ? 4 : 0)};
        blocks += b;
    }
    t.blocks = static_cast<int>(blocks);
    t.per = static_cast<int>((blocks + CTAS - 1) / CTAS);
}
template <int N>
unsigned grid_of(const GradTable<N>& t) { return static_cast<unsigned>((t.blocks + t.per - 1) / t.per); }

int64_t tensors_of(int64_t n, const sdm_grad_tensor* t) {
    int64_t some = 0;
    for (int64_t i = 0; i < n; ++i) some += t[i].n > 0;
    return some;
}

template <int N>
cudaError_t run(int64_t n, const sdm_grad_tensor* list, bool write, float max_norm, float* stats, double* part, cudaStream_t stream) {
    GradTable<N> t;
    int64_t shares = 0;
    bool one = false;                            // table: it still stands for the second pass
    for (int64_t i = 0; i < n;) {
        fill(t, n, list, i);
        if (t.count == 0) break;
        one = shares == 0 && i == n;
        k_grad_squares<N><<<grid_of(t), GT, 0, stream>>>(t, part + shares * 3);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        shares += grid_of(t);
    }
    const int s = static_cast<int>(shares);
    if (!write || shares == 0) {
        k_grad_norm<<<1, GT, 0, stream>>>(part, s, max_norm, stats);
        return cudaGetLastError();
    }
    for (int64_t i = 0; i < n;) {
        if (one) i = n;
        else fill(t, n, list, i);
        if (t.count == 0) break;
        k_grad_scale<N><<<grid_of(t), GT, 0, stream>>>(t, part, s, max_norm, stats);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

// A share is three sums in 64 bits; a launch has at most CTAS of them, and no more than blocks.
size_t grad_bytes(int64_t n, const sdm_grad_tensor* t) {
    size_t blocks = 0;
    for (int64_t i = 0; i < n; ++i) blocks += static_cast<size_t>(blocks_of(t[i]));
    const size_t shares = (static_cast<size_t>(tensors_of(n, t)) + MANY - 1) / MANY * CTAS;
    return (blocks < shares ? blocks : shares) * 3 * 8;
}

cudaError_t launch_grad(int64_t n, const sdm_grad_tensor* list, bool write, float max_norm, float* stats, void* ws, cudaStream_t stream) {
    return tensors_of(n, list) <= FEW ? run<FEW>(n, list, write, max_norm, stats, static_cast<double*>(ws), stream)
                                      : run<MANY>(n, list, write, max_norm, stats, static_cast<double*>(ws), stream);
}

}  // namespace sdm
