// Linear attention with a decay per head: what the C ABI hands to the kernels.
#pragma once
#include "gdn_internal.h"
#include "sdm_common.cuh"

namespace sdm {

constexpr int DLA_C32 = 32;               // tokens per chunk of the fp32 walk
constexpr int DLA_ROLES = 6;              // walks of a call at once: up to three, each in up to two pieces of the contraction

// One walk over the tokens of every (sequence, head): with a state S [da, db] and, for each token in the walk's order,
// operands r and k [da] and v [db] and an output o [db],
//   forwards   S = lam S + add k v^T;  o = S-part: inter S^T r, own chunk: intra (r.k_j) lam^(i - j) v_j
//   backwards  the state is read before the token's own decay and after it only through the token itself.
// The forward pass is one such walk, the backward pass three:
//   y: r = q, k = k, v = v;  dq: r = dy, k = v, v = k on S^T;
//   dv: backwards, r = k, k = q, v = dy on R = dL/dS;  dk: backwards, r = v, k = dy, v = q on R^T.
struct DlaRole {
    const void* r; const void* k; const void* v;
    void* out;
    int hr, hk, hv;           // heads of r, k and v (H or H_k)
    int da, db;
    int x0, width;            // its values of r and k: [x0, x0 + da) of `width` (all, or where the scan cuts them, up to 128)
    const float* state_in;    // [slots, H, d_k, d_v], or nullptr (zero)
    float* state_out;         // or nullptr; may be state_in
    int transposed;           // r and k have width d_v
    int reverse;
    int partial;              // out is float32 [B, H, T, db], a share of the output: of one value head, of some of r's values
    float inter, intra, add;
};
struct DlaWalk {
    int B, H, T, token_major;
    int scan;                 // on the tensor cores
    const float* log_decay;   // [H]
    const int32_t* lengths;   // [B] or nullptr
    int* err;
    int roles;
    DlaRole role[DLA_ROLES];
    int slices[DLA_ROLES];    // of db, a CTA each
    // The tokens may be cut into `segs` pieces of `seg_chunks` chunks that run at once: a first launch copies the first
    // state and takes what each piece but the last adds to it into seg_state [role][B * H][segs][width * db], a small one turns
    // that into the states that the pieces start from, and the walk proper takes them.  The decays over the pieces, in seg_pow
    // [role][B * H][3]: a whole one, the first, the last that has tokens.
    int segs, seg_chunks;
    float2* seg_pow;
    // Or the scan spreads more chains than SMs evenly over these: a list of all chains' chunks, one chain after the other, is cut
    // every `span` chunks (0: it is not).  A chain that is cut hands its state over in seg_state.
    int span;
    int cut_polls;            // of the hand-over, before its wait gives up
    int cut_hold;             // test hook: no state is handed over
    float* seg_state;
    int64_t seg_role[DLA_ROLES];      // where a role's sums start, in floats
};

// lam^n for lam = exp(ld): 1 at n = 0 whatever ld is, 0 for ld = -inf.  The product is taken in two parts.
__device__ __forceinline__ float dla_pow(float ld, int n) {
    if (n == 0) return 1.f;
    const float f = static_cast<float>(n), hi = f * ld, e = expf(hi);
    if (!gdn_finite(hi) || !gdn_finite(e)) return e;
    return fmaf(e, fmaf(f, ld, -hi), e);
}
// The same as two floats: multiplied on once a chunk, a factor that is off by 2^-25 would be off by as much again every time.
__device__ __forceinline__ float2 dla_pow2(float ld, int n) {
    const double f = n == 0 ? 1.0 : exp(static_cast<double>(n) * static_cast<double>(ld));
    const float hi = static_cast<float>(f);
    return make_float2(hi, gdn_finite(hi) ? static_cast<float>(f - static_cast<double>(hi)) : 0.f);
}
// The decays over the pieces of a walk, in two parts (they are multiplied on once a piece); C tokens a chunk, which = 0, 1, 2.
__device__ __forceinline__ void dla_piece_pow(const DlaWalk& w, int role, int64_t chain, float ld, int len, int C, int which) {
    const int chunks = (len + C - 1) / C, s = which == 1 ? 0 : max(0, (chunks - 1) / w.seg_chunks);
    const int s0 = min(s * w.seg_chunks, chunks), s1 = min(s0 + w.seg_chunks, chunks);
    int n = (s1 - s0) * C;                                   // the walk's partial chunk is the sequence's last
    if (s0 < s1 && (w.role[role].reverse ? s0 == 0 : s1 == chunks)) n -= chunks * C - len;
    w.seg_pow[(role * static_cast<int64_t>(w.B) * w.H + chain) * 3 + which] = dla_pow2(ld, which == 0 ? w.seg_chunks * C : n);
}
__device__ __forceinline__ int dla_length(const DlaWalk& w, int b) {
    if (w.lengths == nullptr) return w.T;
    const int n = __ldg(w.lengths + b);
    if (n < 0 || n > w.T) {
        if (threadIdx.x == 0) flag_error(w.err, ERR_BAD_INDEX);
        return n < 0 ? 0 : w.T;
    }
    return n;
}

// Zeros in columns [col0, col0 + cols) of the outputs of tokens `from` and on, in pieces of 16 bytes; every segment's CTA writes
// its share.
template <class D>
__device__ __forceinline__ void dla_zero_tail(const DlaWalk& w, const DlaRole& ro, int b, int h, int col0, int cols, int from, int seg, int tid, int threads) {
    const int es = ro.partial ? 4 : D::BYTES, pieces = cols * es / 16, each = (w.T - from + w.segs - 1) / w.segs;
    const int t0 = from + seg * each, t1 = t0 + each < w.T ? t0 + each : w.T;
    if (t0 >= t1) return;
    const int64_t stride = ro.partial ? ro.db : gdn_stride(w.token_major, w.H, ro.db);
    const int64_t base = ro.partial ? (static_cast<int64_t>(b) * w.H + h) * w.T * ro.db : gdn_base(w.token_major, b, h, w.H, w.T, ro.db);
    char* const out = static_cast<char*>(ro.out) + (base + col0) * es;
    const int rows = threads / pieces, row = tid / pieces;       // rows at once
    if (row >= rows) return;
    for (int64_t t = t0 + row; t < t1; t += rows)
        *reinterpret_cast<uint4*>(out + t * stride * es + tid % pieces * 16) = make_uint4(0, 0, 0, 0);
}

// Fills in segs and seg_chunks; runs the walks.
void dla_plan(DlaWalk& w);
cudaError_t launch_dla(int dtype, DlaWalk& w, cudaStream_t stream);
// The walks on the tensor cores (k_dla_scan.cu): bf16, chunks of 64, da <= 128.
bool dla_scan_pays(int dtype, int T, int dk, int dv);
void dla_scan_plan(DlaWalk& w);
size_t dla_scan_cut_bytes();
int dla_scan_cuts(const DlaWalk& w);              // chains that are cut
cudaError_t launch_dla_scan(DlaWalk& w, cudaStream_t stream);
// The states that the pieces start from, chunks of `chunk` tokens.
cudaError_t launch_dla_prefix(const DlaWalk& w, int chunk, cudaStream_t stream);
// Outputs [heads] that are sums, in order, over `pieces` of the contraction and `group` value heads of their shares
// [pieces][B, heads * group, T, d] float32.
struct DlaSum {
    const float* part;
    void* out;
    int heads, group, pieces, d;
};
struct DlaSums {
    int n;
    DlaSum s[3];
};
cudaError_t launch_dla_join(int dtype, const DlaSums& sums, int B, int T, int token_major, cudaStream_t stream);

struct DlaStep {
    const void* q; const void* k; const void* v;
    const float* log_decay;
    const int32_t* slots;
    float* state;
    void* y;
    int B, H, Hk, dk, dv, n_slots;
    float scale;
    int* err;
};
cudaError_t launch_dla_step(int dtype, const DlaStep& s, cudaStream_t stream);

// ---- block norm (k_block_norm.cu) ----
struct BlockNorm {
    int64_t M, gate_rows;
    int D;
    float eps;
    const void* x; const void* y; const void* gate;                          // forward; backward reads h in place of x
    const float* res_scale; const float* gamma_post; const float* gamma_pre;
    void* h; void* z;                                                        // forward
    const void* dz; const void* dh;                                          // backward
    void* dx; void* dy; void* dgate;
    float* dres_scale; float* dgamma_post; float* dgamma_pre;
    float* ws;
};
bool block_norm_supported(int D);
cudaError_t launch_block_norm(int dtype, const BlockNorm& a, cudaStream_t stream);
size_t block_norm_backward_bytes(int dtype, int64_t M, int64_t gate_rows, int D);
cudaError_t launch_block_norm_backward(int dtype, const BlockNorm& a, cudaStream_t stream);

// ---- gradient norm and clipping (k_grad_clip.cu) ----
size_t grad_bytes(int64_t n, const sdm_grad_tensor* t);
cudaError_t launch_grad(int64_t n, const sdm_grad_tensor* t, bool write, float max_norm, float* stats, void* ws, cudaStream_t stream);

}  // namespace sdm
