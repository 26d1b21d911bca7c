// Gated delta rule (dense state) and linear layer: what the C ABI hands to the kernels.
#pragma once
#include "sdm_internal.h"

#include <atomic>

namespace sdm {

// Tokens per chunk of the saved states: the fp32 kernels and the tensor-core kernels.
constexpr int GDN_C32 = 32;
constexpr int GDN_C64 = 64;

struct GdnArgs {
    const void* q; const void* k;         // [B, Hk, T, dk] or [B, T, Hk, dk]
    const void* v;                        // [B, H, T, dv]  or [B, T, H, dv]
    const void* alpha; const void* beta;  // [B, H, T]
    const int32_t* lengths;               // [B] or nullptr (every sequence has T tokens)
    int B, H, Hk, T, dk, dv;
    int token_major;
    float scale;
    int* err;                             // device status word
};

// Element offset of token 0 and the distance between tokens of one (sequence, head).
__host__ __device__ __forceinline__ int64_t gdn_base(int token_major, int b, int h, int heads, int T, int d) {
    return token_major ? (static_cast<int64_t>(b) * T * heads + h) * d
                       : (static_cast<int64_t>(b) * heads + h) * T * static_cast<int64_t>(d);
}
__host__ __device__ __forceinline__ int64_t gdn_stride(int token_major, int heads, int d) {
    return token_major ? static_cast<int64_t>(heads) * d : d;
}

// Tokens of sequence b; a length outside [0, T] is clamped and recorded in the status word.
__device__ __forceinline__ int gdn_length(const GdnArgs& a, int b) {
    if (a.lengths == nullptr) return a.T;
    const int n = __ldg(a.lengths + b);
    if (n < 0 || n > a.T) {
        if (threadIdx.x == 0) flag_error(a.err, ERR_BAD_INDEX);
        return n < 0 ? 0 : a.T;
    }
    return n;
}

__device__ __forceinline__ bool gdn_finite(float x) { return fabsf(x) <= 3.402823466e+38f; }
__device__ __forceinline__ float gdn_nan() { return __int_as_float(0x7fffffff); }

// Dynamic shared memory above 48 KB has to be allowed once per kernel and device; the call costs about
// as much as a launch, so it is not repeated.
template <class K>
inline cudaError_t allow_smem(K kernel, size_t bytes, std::atomic<unsigned long long>& seen) {
    if (bytes <= 32 * 1024) return cudaSuccess;  // up to 48 KB without leave, static shared memory included
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (bit & seen.load(std::memory_order_acquire)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (e == cudaSuccess) seen.fetch_or(bit, std::memory_order_release);
    return e;
}

// A kernel that splits its registers among its warps takes them out of what the CTA is launched with, so that has to be
// `want` a thread.  `get(int*)` asks for the count once; only an answer is kept, a failure is not.
template <class Get>
inline cudaError_t check_registers(int want, std::atomic<int>& known, Get get) {
    int n = known.load(std::memory_order_acquire);
    if (n == 0) {
        const cudaError_t e = get(&n);
        if (e != cudaSuccess) return e;
        known.store(n, std::memory_order_release);
    }
    return n == want ? cudaSuccess : cudaErrorInvalidConfiguration;
}
template <class K>
inline cudaError_t check_kernel_registers(K kernel, int want, std::atomic<int>& known) {
    return check_registers(want, known, [kernel](int* n) {
        cudaFuncAttributes at;
        const cudaError_t e = cudaFuncGetAttributes(&at, kernel);
        if (e == cudaSuccess) *n = at.numRegs;
        return e;
    });
}

// ---- token recurrence (k_gdn_recur.cu) ----
struct GdnRecur {
    GdnArgs a;
    float* state;             // forward: [slots, H, dk, dv], updated in place (nullptr: see state_in)
    const float* state_in;    // forward with saved states: the initial state (left as it is);
                              // reverse: dL/dS_T or nullptr (zero)
    const int32_t* slots;     // T = 1: [B] row of `state` of each sequence, or nullptr (row b)
    int n_slots;
    void* y;                  // forward: y; reverse: dv
    const void* dy;           // reverse
    float* marks;             // saved states [B, H, ceil(T / 32), dk, dv]: forward, at the start of every
                              // chunk; reverse, the gradient of the state at the end of every chunk
    float* rows;              // forward with saved states: e [B, H, T, dv]; reverse: d
    float* state_out;         // reverse: dL/dS_0 or nullptr
};
// mode 0: forward; 1: forward with saved states and e, no y; 2: reverse.
cudaError_t launch_gdn_recur(int dtype, int mode, const GdnRecur& r, cudaStream_t stream);

// The same walks in chunks of 32 (k_gdn_walk.cu): float32, few chains.  fact: gdn_walk_bytes of scratch.
bool gdn_walk_supported(int dtype, int B, int H, int T, int dv);
size_t gdn_walk_bytes(int64_t chunks);
cudaError_t launch_gdn_walk(int mode, const GdnRecur& r, float* fact, cudaStream_t stream);

// ---- gradients of q, k and the gates from the saved states (k_gdn_grads.cu), chunks of 32 ----
struct GdnGrads {
    GdnArgs a;
    const void* dy;
    const float* S; const float* dE;      // [B, H, nc, dk, dv]
    const float* e; const float* d;       // [B, H, T, dv]
    void* dq; void* dk; void* dalpha; void* dbeta;
};
cudaError_t launch_gdn_grads(int dtype, const GdnGrads& g, cudaStream_t stream);

// ---- chunked form on the tensor cores (k_gdn_chunk.cu): bf16, d_k <= 128, chunks of 64 ----
// What the chunks' own products are, per (sequence, head, chunk): bf16 matrices [64][64], N as three parts (24
// significant bits), then P as two, or for the backward, whose state depends on it, as three; and three rows of 64 floats.
constexpr int GDN_N_PARTS = 3, GDN_SCAN_MATS = GDN_N_PARTS + 2, GDN_BACK_MATS = GDN_N_PARTS + 3;
struct GdnFactors {
    void* mat;                // [B, H, nc, mats, 64, 64] bf16
    int mats;                 // GDN_SCAN_MATS, or for the backward GDN_BACK_MATS
    float* gates;             // [B, H, nc, 3, 64]: prod_{l <= i} alpha_l, beta_i, prod_{l > i} alpha_l.  From a chunk's first
                              // token on whose k, alpha or beta is not finite, the first are not, and N, P and beta are 0
};
size_t gdn_factor_mat_bytes(int64_t chunks, int mats);
size_t gdn_factor_gate_bytes(int64_t chunks);
bool gdn_chunk_supported(int dtype, int dk, int T);
cudaError_t launch_gdn_factors(const GdnArgs& a, const GdnFactors& f, cudaStream_t stream);
struct GdnScan {
    GdnArgs a;
    float* state;             // [B, H, dk, dv], updated in place
    void* y;
    const float* state_in;    // with keep_S: the first state, left as it is
    void* keep_S;             // [B, H, nc, dv', dk'] bf16: the states before the chunks, transposed, or nullptr
                              // (dv': d_v rounded up to 128, dk': d_k to 64 or 128)
    void* keep_e;             // [B, H, nc, 2, dv', 64] bf16: e as upper and lower parts, transposed
};
cudaError_t launch_gdn_scan(const GdnScan& s, const GdnFactors& f, cudaStream_t stream);

// The backward's walk (k_gdn_back.cu), with f.mats == GDN_BACK_MATS.
struct GdnBack {
    GdnArgs a;
    const void* dy;
    const float* dstate;      // dL/dS_T or nullptr (zero)
    void* dv;
    float* dstate0;           // dL/dS_0 or nullptr
    void* keep_D;             // [B, H, nc, dv', dk'] bf16: the gradients of the states after the chunks, transposed
    void* keep_d;             // [B, H, nc, 2, dv', 64] bf16: d as upper and lower parts, transposed
    const void* e;            // as the forward walk stored it (GdnScan::keep_e)
    float* ke;                // [B, H, nc, dv' / 32, 64]: <D^T k_j, e_j> over 32 columns, D after the chunk
};
cudaError_t launch_gdn_back(const GdnBack& r, const GdnFactors& f, cudaStream_t stream);

// Gradients of q, k and the gates from what the two walks stored (k_gdn_grads_tc.cu).
struct GdnGradsTc {
    GdnArgs a;
    const void* dy;
    const float* gates;       // GdnFactors::gates
    const void* S; const void* D; const void* e; const void* d; const float* ke;   // as GdnScan and GdnBack store them
    void* dq; void* dk; void* dalpha; void* dbeta;
};
cudaError_t launch_gdn_grads_tc(const GdnGradsTc& g, cudaStream_t stream);

// ---- linear layer (k_linear.cu): bf16 matrices, row-major ----
// out [M, N] = residual + act(x W^T + bias); pre (optional) receives x W^T + bias.
struct LinearOut {
    const float* bias;                    // [N] or nullptr
    const void* residual;                 // [M, N] bf16 or nullptr
    void* pre;                            // [M, N] bf16 or nullptr
    void* out;                            // [M, N] bf16
    int act;
};
// How a product is cut: 128 x bn tiles, `splits` ranges of the contraction (each a multiple of 64)
// whose fp32 shares are joined by a second kernel.
struct LinearPlan {
    int bn, splits;
};
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K);
size_t linear_split_bytes(int64_t M, int64_t N, int64_t K);
bool linear_skinny(int64_t M);
// D[m, n] = sum_k A(m, k) B(n, k).  A is [M, K] (a_mn = false) or [K, M] in memory; B alike.
cudaError_t launch_linear(const void* A, bool a_mn, const void* B, bool b_mn, int64_t M, int64_t N, int64_t K,
                          const LinearOut& o, float* split_ws, int* err, cudaStream_t stream);
cudaError_t launch_linear_skinny(const void* x, const void* W, int M, int N, int K, const LinearOut& o,
                                 cudaStream_t stream);
// dp = dout act'(pre) (dp == nullptr: not written) and dbias = column sums of it (nullptr: not
// taken); part: linear_dact_bytes(M, N) of scratch for the column sums.
size_t linear_dact_bytes(int64_t M, int64_t N);
cudaError_t launch_linear_dact(const void* dout, const void* pre, int act, int64_t M, int N, void* dp, float* dbias,
                               float* part, cudaStream_t stream);

}  // namespace sdm
