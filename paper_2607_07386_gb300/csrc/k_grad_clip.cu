// The global norm of many gradients, and clipping by it:
//   norm = sqrt(sum over all tensors of g^2),  out = g min(1, max_norm / norm).
//
// Bound by memory: one pass reads everything for the norm, the second reads it again and writes.  The second walks the
// blocks backwards, so that what the first read last is still in L2.
//
// The list goes to the kernels in their parameters (TABLE tensors a launch): nothing is copied to the device first, and a
// captured launch holds its list.  A CTA takes blocks of BLOCK bytes of one tensor; its sums go to the workspace, and
// are joined in order, so the norm is the same on every call.
//
// Squares of float32 values run out of float32's range at 2^64 and 2^-63, long before the values do, so three sums are kept:
// of x^2, (2^-80 x)^2 and (2^80 x)^2.  The joining kernel takes the first unless it overflowed or is so small that
// squares were lost.
#include "dla_internal.h"
#include "sdm_common.cuh"

namespace sdm {

namespace {

constexpr int GT = 256, PIECES = 8;              // threads; pieces of 16 bytes of the gradient a thread
constexpr int64_t BLOCK = GT * PIECES * 16;      // bytes of the gradient a block
constexpr int TABLE = 120;

struct GradTable {
    const void* src[TABLE];
    void* dst[TABLE];
    int64_t n[TABLE];
    int first[TABLE + 1];                        // the tensor's first block of this launch
    unsigned char kind[TABLE];                   // bit 0: src is bf16; bit 1: dst is bf16; bit 2: one by one (addresses that do not match)
    int count;
};
static_assert(sizeof(GradTable) <= 3900, "kernel parameters");

template <bool B> struct Type { using D = F32; };
template <> struct Type<true> { using D = BF16; };

__device__ __forceinline__ int find(const GradTable& t, int block) {
    int lo = 0, hi = t.count;                    // first[lo] <= block < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}
constexpr float UP = 1208925819614629174706176.f, DOWN = 1.f / UP;      // 2^80

__device__ __forceinline__ void add_square(float x, float (&s)[3]) {
    const float d = x * DOWN, u = x * UP;
    s[0] = fmaf(x, x, s[0]);
    s[1] = fmaf(d, d, s[1]);
    s[2] = fmaf(u, u, s[2]);
}

// Elements of a tensor before its first 16-byte boundary (all of them are whole elements away from it).
template <class D> __device__ __forceinline__ int head_of(const void* p, int64_t n) {
    const int h = static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / D::BYTES;
    return h < n ? h : static_cast<int>(n);
}

template <class D>
__device__ __forceinline__ void squares(const void* src, int64_t n, int64_t block, float (&s)[3]) {
    using T = typename D::T;
    const T* p = static_cast<const T*>(src);
    const int head = head_of<D>(src, n);
    const int64_t pieces = (n - head) / D::E, first = block * (GT * PIECES) + threadIdx.x;
    const uint4* v = reinterpret_cast<const uint4*>(p + head);
    uint4 u[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) u[i] = first + i * GT < pieces ? __ldg(v + first + i * GT) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        float f[8];
        unpack16<D>(u[i], f);
#pragma unroll
        for (int e = 0; e < D::E; ++e) add_square(f[e], s);
    }
    if (block == 0) {                            // what lies before and behind the pieces
        const int64_t tail = head + pieces * D::E;
        if (threadIdx.x < head) add_square(load_elem<D>(src, threadIdx.x), s);
        if (tail + threadIdx.x < n) add_square(load_elem<D>(src, tail + threadIdx.x), s);
    }
}

__global__ void __launch_bounds__(GT) k_grad_squares(const __grid_constant__ GradTable t, float* __restrict__ part) {
    __shared__ float sh[GT / 32][3];
    const int at = find(t, blockIdx.x);
    float s[3] = {0.f, 0.f, 0.f};
    if (t.kind[at] & 1) squares<BF16>(t.src[at], t.n[at], blockIdx.x - t.first[at], s);
    else squares<F32>(t.src[at], t.n[at], blockIdx.x - t.first[at], s);
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) {
        sh[warp][0] = s[0];
        sh[warp][1] = s[1];
        sh[warp][2] = s[2];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        float x = 0.f;
        for (int w = 0; w < GT / 32; ++w) x += sh[w][threadIdx.x];
        part[static_cast<int64_t>(blockIdx.x) * 3 + threadIdx.x] = x;
    }
}

// The norm and the factor from the blocks' sums, in 64 bits and in order.
__global__ void __launch_bounds__(1024) k_grad_norm(const float* __restrict__ part, int64_t blocks, float max_norm, float* __restrict__ stats) {
    __shared__ double sh[32][3];
    double s[3] = {0, 0, 0};
    for (int64_t i = threadIdx.x; i < blocks; i += 1024)
#pragma unroll
        for (int j = 0; j < 3; ++j) s[j] += __ldg(part + i * 3 + j);
#pragma unroll
    for (int j = 0; j < 3; ++j)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0)
        for (int j = 0; j < 3; ++j) sh[warp][j] = s[j];
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int j = 0; j < 3; ++j) {
        s[j] = 0;
        for (int w = 0; w < 32; ++w) s[j] += sh[w][j];
    }
    const double big = 3.4e38, small = 1e-20;    // below, squares of 2^-63 and less may have counted
    double norm = s[0] <= big && s[0] >= small ? sqrt(s[0]) : s[0] < small ? sqrt(s[2]) * static_cast<double>(DOWN) : sqrt(s[1]) * static_cast<double>(UP);
    if (s[0] != s[0]) norm = s[0];
    const float f = static_cast<float>(norm);
    stats[0] = f;
    stats[1] = !(fabsf(f) <= 3.402823466e+38f) ? __int_as_float(0x7fffffff) : norm > max_norm ? static_cast<float>(max_norm / norm) : 1.f;
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
__device__ __forceinline__ void scale(const void* src, void* dst, int64_t n, int64_t block, bool singly, float f) {
    if (singly) {
        const int64_t per = GT * PIECES * S::E, first = block * per;
        const int64_t last = first + per < n ? first + per : n;
        for (int64_t i = first + threadIdx.x; i < last; i += GT) put_elem<S, O>(src, dst, i, f);
        return;
    }
    const int head = head_of<S>(src, n);
    const int64_t pieces = (n - head) / S::E, first = block * (GT * PIECES) + threadIdx.x;
    const uint4* v = reinterpret_cast<const uint4*>(static_cast<const typename S::T*>(src) + head);
    uint4 u[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) u[i] = first + i * GT < pieces ? __ldcs(v + first + i * GT) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        if (first + i * GT >= pieces) break;
        if (S::BYTES == O::BYTES && f == 1.f) {
            *reinterpret_cast<uint4*>(static_cast<typename O::T*>(dst) + head + (first + i * GT) * S::E) = u[i];
            continue;
        }
        float x[8];
        unpack16<S>(u[i], x);
#pragma unroll
        for (int e = 0; e < S::E; ++e) x[e] *= f;
        put_piece<S, O>(dst, head + (first + i * GT) * S::E, x);
    }
    if (block == 0) {
        const int64_t tail = head + pieces * S::E;
        if (threadIdx.x < head) put_elem<S, O>(src, dst, threadIdx.x, f);
        if (tail + threadIdx.x < n) put_elem<S, O>(src, dst, tail + threadIdx.x, f);
    }
}

__global__ void __launch_bounds__(GT) k_grad_scale(const __grid_constant__ GradTable t, const float* __restrict__ stats) {
    const int block = gridDim.x - 1 - blockIdx.x;
    const int at = find(t, block);
    float f = __ldg(stats + 1);
    if (f != f) f = 1.f;                         // the norm is not finite: the gradients stay as they are
    const int kind = t.kind[at];
    const void* src = t.src[at];
    void* dst = t.dst[at];
    if (f == 1.f && src == dst) return;
    const int64_t n = t.n[at], b = block - t.first[at];
    const bool singly = kind & 4;
    switch (kind & 3) {
        case 0: scale<F32, F32>(src, dst, n, b, singly, f); break;
        case 1: scale<BF16, F32>(src, dst, n, b, singly, f); break;
        case 2: scale<F32, BF16>(src, dst, n, b, singly, f); break;
        default: scale<BF16, BF16>(src, dst, n, b, singly, f); break;
    }
}

int64_t blocks_of(const sdm_grad_tensor& t) {
    const int64_t bytes = t.n * (t.dtype == SDM_F32 ? 4 : 2);
    return (bytes + BLOCK - 1) / BLOCK;
}
// The next launch's table; `i` goes past what it took.
int64_t fill(GradTable& t, int64_t n, const sdm_grad_tensor* list, int64_t& i) {
    t.count = 0;
    int64_t blocks = 0;
    for (; i < n && t.count < TABLE; ++i) {
        const sdm_grad_tensor& g = list[i];
        const int64_t b = blocks_of(g);
        if (b == 0) continue;
        if (blocks + b > INT32_MAX) break;
        const int k = t.count++;
        t.src[k] = g.grad;
        t.dst[k] = g.out;
        t.n[k] = g.n;
        t.first[k] = static_cast<int>(blocks);
        const bool half = g.dtype == SDM_BF16, out_half = g.out_dtype == SDM_BF16;
        // the pieces of src begin on 16 bytes; those of dst must begin on their own size
        const uintptr_t s = reinterpret_cast<uintptr_t>(g.grad), d = reinterpret_cast<uintptr_t>(g.out);
        const uintptr_t head = ((16 - s % 16) % 16) / (half ? 2 : 4) * (out_half ? 2 : 4);
        const uintptr_t need = !half && out_half ? 8 : 16;
        t.kind[k] = static_cast<unsigned char>((half ? 1 : 0) | (out_half ? 2 : 0) | ((d + head) % need != 0 ? 4 : 0));
        blocks += b;
    }
    t.first[t.count] = static_cast<int>(blocks);
    return blocks;
}

}  // namespace

size_t grad_bytes(int64_t n, const sdm_grad_tensor* t) {
    size_t blocks = 0;
    for (int64_t i = 0; i < n; ++i) blocks += static_cast<size_t>(blocks_of(t[i]));
    return blocks * 3 * 4;
}

cudaError_t launch_grad(int64_t n, const sdm_grad_tensor* list, bool write, float max_norm, float* stats, void* ws, cudaStream_t stream) {
    GradTable t;
    float* const part = static_cast<float*>(ws);
    int64_t done = 0;
    for (int64_t i = 0; i < n;) {
        const int64_t blocks = fill(t, n, list, i);
        if (blocks == 0) break;
        k_grad_squares<<<static_cast<unsigned>(blocks), GT, 0, stream>>>(t, part + done * 3);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        done += blocks;
    }
    k_grad_norm<<<1, 1024, 0, stream>>>(part, done, max_norm, stats);
    cudaError_t e = cudaGetLastError();
    if (!write) return e;
    for (int64_t i = 0; i < n && e == cudaSuccess;) {
        const int64_t blocks = fill(t, n, list, i);
        if (blocks == 0) break;
        k_grad_scale<<<static_cast<unsigned>(blocks), GT, 0, stream>>>(t, stats);
        e = cudaGetLastError();
    }
    return e;
}

}  // namespace sdm
