// C ABI of the gated delta rule and the linear layer: argument checks, workspaces, launches.
// Declarations and semantics: include/sdm.h.
#include "api_check.h"
#include "gdn_internal.h"

static_assert(sizeof(sdm_gdn_shape) == 36, "sdm_gdn_shape layout is part of the ABI");
static_assert(sizeof(sdm_linear_shape) == 24, "sdm_linear_shape layout is part of the ABI");

namespace {

// ------------------------------------------------------------------ gated delta rule
sdm_status gdn_check(const sdm_gdn_shape* s) {
    if (!s) return fail(SDM_ERR_INVALID_ARG, "shape is NULL");
    if (s->B < 0 || s->H < 0 || s->T < 0) return fail(SDM_ERR_INVALID_ARG, "B, H, T must be >= 0 (got %d, %d, %d)", s->B, s->H, s->T);
    if (s->B > 65535 || s->H > 65535) return fail(SDM_ERR_UNSUPPORTED, "B and H must be <= 65535 (got %d, %d)", s->B, s->H);
    if (s->T > INT_MAX - 64) return fail(SDM_ERR_UNSUPPORTED, "T too large (%d)", s->T);
    if (s->H > 0 && (s->H_k < 1 || s->H % s->H_k != 0))
        return fail(SDM_ERR_INVALID_ARG, "H must be a multiple of H_k >= 1 (got %d, %d)", s->H, s->H_k);
    if (s->dtype != SDM_F32 && s->dtype != SDM_BF16) return fail(SDM_ERR_INVALID_ARG, "unknown dtype %d", s->dtype);
    if (s->layout != SDM_HEAD_MAJOR && s->layout != SDM_TOKEN_MAJOR) return fail(SDM_ERR_INVALID_ARG, "unknown layout %d", s->layout);
    if (s->d_k < 1 || s->d_v < 1) return fail(SDM_ERR_INVALID_ARG, "d_k and d_v must be >= 1 (got %d, %d)", s->d_k, s->d_v);
    if (s->d_k > 256) return fail(SDM_ERR_UNSUPPORTED, "d_k > 256 is not supported (d_k=%d)", s->d_k);
    if (s->d_v > (1 << 20)) return fail(SDM_ERR_UNSUPPORTED, "d_v too large (%d)", s->d_v);
    if (static_cast<int64_t>(s->B) * s->H * ((static_cast<int64_t>(s->T) + 63) / 64) > INT_MAX / 256 / ((s->d_v + 127) / 128))
        return fail(SDM_ERR_UNSUPPORTED, "B * H * T / 64 * d_v / 128 must be below 2^23 (got %d, %d, %d, %d)", s->B, s->H, s->T, s->d_v);
    const size_t es = esize(s->dtype);
    if (s->d_k * es % 16 != 0 || s->d_v * es % 16 != 0)
        return fail(SDM_ERR_UNSUPPORTED, "d_k and d_v times the element size must be multiples of 16 bytes (d_k=%d, d_v=%d)", s->d_k, s->d_v);
    if (!(s->scale - s->scale == 0.f)) return fail(SDM_ERR_INVALID_ARG, "scale must be finite");
    return SDM_OK;
}

struct GdnSizes {
    size_t qk, v, gate, state, es;
};
GdnSizes gdn_sizes(const sdm_gdn_shape* s) {
    const size_t es = esize(s->dtype), bt = static_cast<size_t>(s->B) * s->T;
    return GdnSizes{bt * s->H_k * s->d_k * es, bt * s->H * s->d_v * es, bt * s->H * es,
                    static_cast<size_t>(s->B) * s->H * s->d_k * s->d_v * 4, es};
}

sdm::GdnArgs gdn_args(const sdm_gdn_shape* s, const void* q, const void* k, const void* v, const void* alpha,
                      const void* beta, const int32_t* lengths, int* err) {
    sdm::GdnArgs a{};
    a.q = q; a.k = k; a.v = v; a.alpha = alpha; a.beta = beta; a.lengths = lengths;
    a.B = s->B; a.H = s->H; a.Hk = s->H_k; a.T = s->T; a.dk = s->d_k; a.dv = s->d_v;
    a.token_major = s->layout == SDM_TOKEN_MAJOR;
    a.scale = s->scale;
    a.err = err;
    return a;
}

// Factors of the chunked forms: bf16 matrices and gate products, or fp32 factors.
struct FwdLayout {
    size_t mat, gates, total;
    bool tc;
};
size_t walk_bytes(const sdm_gdn_shape* s) {
    if (!sdm::gdn_walk_supported(s->dtype, s->B, s->H, s->T, s->d_v)) return 0;
    return align256(sdm::gdn_walk_bytes(static_cast<int64_t>(s->B) * s->H * ((s->T + sdm::GDN_C32 - 1) / sdm::GDN_C32)));
}
FwdLayout fwd_layout(const sdm_gdn_shape* s) {
    FwdLayout L{};
    L.tc = sdm::gdn_chunk_supported(s->dtype, s->d_k, s->T);
    if (!L.tc) {
        L.total = walk_bytes(s);
        return L;
    }
    const int64_t chunks = static_cast<int64_t>(s->B) * s->H * ((s->T + sdm::GDN_C64 - 1) / sdm::GDN_C64);
    L.gates = align256(sdm::gdn_factor_mat_bytes(chunks, sdm::GDN_SCAN_MATS));
    L.total = L.gates + align256(sdm::gdn_factor_gate_bytes(chunks));
    return L;
}

// What the walks of the backward store: the fp32 kernels states and rows, the tensor-core kernels the
// chunks' factors, then states and rows as bf16 (see GdnScan, GdnBack).
struct BwdLayout {
    bool tc;
    size_t mat, gates, S, dE, e, d, ke, fact, total;
};
BwdLayout bwd_layout(const sdm_gdn_shape* s) {
    BwdLayout L{};
    const size_t bh = static_cast<size_t>(s->B) * s->H, T = static_cast<size_t>(s->T);
    L.tc = sdm::gdn_chunk_supported(s->dtype, s->d_k, s->T);
    size_t marks, rows, ke = 0;
    if (L.tc) {
        const size_t chunks = bh * ((T + sdm::GDN_C64 - 1) / sdm::GDN_C64), dvp = (static_cast<size_t>(s->d_v) + 127) / 128 * 128;
        L.gates = align256(sdm::gdn_factor_mat_bytes(static_cast<int64_t>(chunks), sdm::GDN_BACK_MATS));
        L.S = L.gates + align256(sdm::gdn_factor_gate_bytes(static_cast<int64_t>(chunks)));
        marks = chunks * dvp * (s->d_k <= 64 ? 64 : 128) * 2;
        rows = chunks * 2 * dvp * sdm::GDN_C64 * 2;
        ke = chunks * (dvp / 32) * sdm::GDN_C64 * 4;
    } else {
        marks = bh * ((T + sdm::GDN_C32 - 1) / sdm::GDN_C32) * s->d_k * s->d_v * 4;
        rows = bh * T * s->d_v * 4;
    }
    L.dE = L.S + align256(marks);
    L.e = L.dE + align256(marks);
    L.d = L.e + align256(rows);
    L.ke = L.d + align256(rows);
    L.fact = L.ke + align256(ke);
    L.total = L.fact + (L.tc ? 0 : walk_bytes(s));
    return L;
}

// ------------------------------------------------------------------ linear layer
sdm_status linear_check(const sdm_linear_shape* s) {
    if (!s) return fail(SDM_ERR_INVALID_ARG, "shape is NULL");
    if (s->M < 0 || s->N < 1 || s->K < 1) return fail(SDM_ERR_INVALID_ARG, "M must be >= 0, N and K >= 1 (got %lld, %d, %d)", (long long)s->M, s->N, s->K);
    if (s->N % 8 != 0 || s->K % 8 != 0) return fail(SDM_ERR_UNSUPPORTED, "N and K must be multiples of 8 (got %d, %d)", s->N, s->K);
    if (s->M > (1 << 24) - 256 || s->N > (1 << 24) - 256 || s->K > (1 << 24) - 256)
        return fail(SDM_ERR_UNSUPPORTED, "M, N and K must be at most 2^24 - 256 (got %lld, %d, %d)", (long long)s->M, s->N, s->K);
    if (s->act < SDM_ACT_NONE || s->act > SDM_ACT_GELU) return fail(SDM_ERR_INVALID_ARG, "unknown activation %d", s->act);
    const int64_t tiles = ((s->M + 127) / 128) * ((s->N + 63) / 64), tx = ((s->M + 127) / 128) * ((s->K + 63) / 64),
                  tw = ((static_cast<int64_t>(s->N) + 127) / 128) * ((s->K + 63) / 64);
    if (tiles > (1 << 26) || tx > (1 << 26) || tw > (1 << 26)) return fail(SDM_ERR_UNSUPPORTED, "the product has too many tiles");
    return SDM_OK;
}

size_t linear_fwd_ws(const sdm_linear_shape* s) {
    return s->M == 0 || sdm::linear_skinny(s->M) ? 0 : align256(sdm::linear_split_bytes(s->M, s->N, s->K));
}
struct LinearBwdLayout {
    size_t dp, part, split, total;
};
LinearBwdLayout linear_bwd_layout(const sdm_linear_shape* s) {
    LinearBwdLayout L{};
    const size_t sx = sdm::linear_split_bytes(s->M, s->K, s->N), sw = sdm::linear_split_bytes(s->N, s->K, s->M);
    L.dp = 0;
    L.part = s->act == SDM_ACT_NONE ? 0 : align256(static_cast<size_t>(s->M) * s->N * 2);
    L.split = L.part + align256(sdm::linear_dact_bytes(s->M, s->N));
    L.total = L.split + align256(sx > sw ? sx : sw);
    return L;
}

}  // namespace

extern "C" {

size_t sdm_gdn_workspace_bytes(const sdm_gdn_shape* s) {
    if (gdn_check(s) != SDM_OK) return 0;
    sdm::api_ok();
    return fwd_layout(s).total;
}

size_t sdm_gdn_backward_workspace_bytes(const sdm_gdn_shape* s) {
    if (gdn_check(s) != SDM_OK) return 0;
    sdm::api_ok();
    return bwd_layout(s).total;
}

sdm_status sdm_gdn_forward(const sdm_gdn_shape* s, const void* q, const void* k, const void* v, const void* alpha,
                           const void* beta, const int32_t* lengths, float* state, void* y, void* workspace,
                           size_t workspace_bytes, sdm_stream_t stream) {
    SDM_TRY(gdn_check(s));
    const GdnSizes z = gdn_sizes(s);
    if (static_cast<size_t>(s->B) * s->H * s->T == 0) return sdm::api_ok();
    const FwdLayout L = fwd_layout(s);
    const size_t need = L.total;
    const Buf bufs[] = {{"q", q, z.qk, 16, false, false}, {"k", k, z.qk, 16, false, false}, {"v", v, z.v, 16, false, false},
                        {"alpha", alpha, z.gate, z.es, false, false}, {"beta", beta, z.gate, z.es, false, false},
                        {"lengths", lengths, static_cast<size_t>(s->B) * 4, 4, true, false},
                        {"state", state, z.state, 16, false, true}, {"y", y, z.v, 16, false, true},
                        {"workspace", workspace, need, 16, true, true}};
    SDM_TRY(check_bufs("sdm_gdn_forward", bufs, 9));
    SDM_TRY(check_ws("sdm_gdn_forward", workspace, workspace_bytes, need));
    int* err = nullptr;
    SDM_TRY(sdm::api_status_word(&err));
    const sdm::GdnArgs a = gdn_args(s, q, k, v, alpha, beta, lengths, err);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (L.tc) {
        char* ws = static_cast<char*>(workspace);
        const sdm::GdnFactors f{ws + L.mat, sdm::GDN_SCAN_MATS, reinterpret_cast<float*>(ws + L.gates)};
        cudaError_t e = sdm::launch_gdn_factors(a, f, st);
        if (e == cudaSuccess) e = sdm::launch_gdn_scan(sdm::GdnScan{a, state, y, nullptr, nullptr, nullptr}, f, st);
        return done(e, "sdm_gdn_forward");
    }
    sdm::GdnRecur r{};
    r.a = a;
    r.state = state;
    r.n_slots = s->B;
    r.y = y;
    return done(L.total > 0 ? sdm::launch_gdn_walk(0, r, static_cast<float*>(workspace), st)
                            : sdm::launch_gdn_recur(s->dtype, 0, r, st), "sdm_gdn_forward");
}

sdm_status sdm_gdn_step(const sdm_gdn_shape* s, const void* q, const void* k, const void* v, const void* alpha,
                        const void* beta, const int32_t* slots, int32_t n_slots, float* state, void* y, sdm_stream_t stream) {
    SDM_TRY(gdn_check(s));
    if (s->T != 1) return fail(SDM_ERR_INVALID_ARG, "sdm_gdn_step needs shape->T == 1 (got %d)", s->T);
    if (n_slots < 0 || (slots == nullptr && n_slots < s->B))
        return fail(SDM_ERR_INVALID_ARG, "sdm_gdn_step: n_slots = %d for B = %d sequences", n_slots, s->B);
    const GdnSizes z = gdn_sizes(s);
    if (static_cast<size_t>(s->B) * s->H == 0) return sdm::api_ok();
    const Buf bufs[] = {{"q", q, z.qk, 16, false, false}, {"k", k, z.qk, 16, false, false}, {"v", v, z.v, 16, false, false},
                        {"alpha", alpha, z.gate, z.es, false, false}, {"beta", beta, z.gate, z.es, false, false},
                        {"slots", slots, static_cast<size_t>(s->B) * 4, 4, true, false},
                        {"state", state, static_cast<size_t>(n_slots) * s->H * s->d_k * s->d_v * 4, 16, false, true},
                        {"y", y, z.v, 16, false, true}};
    SDM_TRY(check_bufs("sdm_gdn_step", bufs, 8));
    int* err = nullptr;
    SDM_TRY(sdm::api_status_word(&err));
    sdm::GdnRecur r{};
    r.a = gdn_args(s, q, k, v, alpha, beta, nullptr, err);
    r.state = state;
    r.slots = slots;
    r.n_slots = n_slots;
    r.y = y;
    return done(sdm::launch_gdn_recur(s->dtype, 0, r, reinterpret_cast<cudaStream_t>(stream)), "sdm_gdn_step");
}

sdm_status sdm_gdn_backward(const sdm_gdn_shape* s, const void* q, const void* k, const void* v, const void* alpha,
                            const void* beta, const int32_t* lengths, const float* state0, const void* dy,
                            const float* dstate, void* dq, void* dk, void* dv, void* dalpha, void* dbeta, float* dstate0,
                            void* workspace, size_t workspace_bytes, sdm_stream_t stream) {
    SDM_TRY(gdn_check(s));
    if (static_cast<size_t>(s->B) * s->H == 0) return sdm::api_ok();
    const GdnSizes z = gdn_sizes(s);
    const BwdLayout L = bwd_layout(s);
    const Buf bufs[] = {{"q", q, z.qk, 16, false, false}, {"k", k, z.qk, 16, false, false}, {"v", v, z.v, 16, false, false},
                        {"alpha", alpha, z.gate, z.es, false, false}, {"beta", beta, z.gate, z.es, false, false},
                        {"lengths", lengths, static_cast<size_t>(s->B) * 4, 4, true, false},
                        {"state0", state0, z.state, 16, false, false}, {"dy", dy, z.v, 16, false, false},
                        {"dstate", dstate, z.state, 16, true, false}, {"dq", dq, z.qk, 16, false, true},
                        {"dk", dk, z.qk, 16, false, true}, {"dv", dv, z.v, 16, false, true},
                        {"dalpha", dalpha, z.gate, z.es, false, true}, {"dbeta", dbeta, z.gate, z.es, false, true},
                        {"dstate0", dstate0, z.state, 16, true, true}, {"workspace", workspace, L.total, 16, true, true}};
    SDM_TRY(check_bufs("sdm_gdn_backward", bufs, 16));
    SDM_TRY(check_ws("sdm_gdn_backward", workspace, workspace_bytes, L.total));
    int* err = nullptr;
    SDM_TRY(sdm::api_status_word(&err));
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    const sdm::GdnArgs a = gdn_args(s, q, k, v, alpha, beta, lengths, err);
    if (L.tc) {
        float* const ke = reinterpret_cast<float*>(ws + L.ke);
        const sdm::GdnFactors fa{ws + L.mat, sdm::GDN_BACK_MATS, reinterpret_cast<float*>(ws + L.gates)};
        cudaError_t e = sdm::launch_gdn_factors(a, fa, st);
        if (e == cudaSuccess) e = sdm::launch_gdn_scan(sdm::GdnScan{a, nullptr, nullptr, state0, ws + L.S, ws + L.e}, fa, st);
        if (e == cudaSuccess) e = sdm::launch_gdn_back(sdm::GdnBack{a, dy, dstate, dv, dstate0, ws + L.dE, ws + L.d, ws + L.e, ke}, fa, st);
        if (e == cudaSuccess)
            e = sdm::launch_gdn_grads_tc(sdm::GdnGradsTc{a, dy, fa.gates, ws + L.S, ws + L.dE, ws + L.e, ws + L.d, ke, dq, dk, dalpha, dbeta}, st);
        return done(e, "sdm_gdn_backward");
    }
    float* const fact = L.total > L.fact ? reinterpret_cast<float*>(ws + L.fact) : nullptr;
    sdm::GdnRecur f{};
    f.a = a;
    sdm::GdnRecur r = f;
    cudaError_t e = cudaSuccess;
    if (s->T > 0) {
        f.state_in = state0;
        f.marks = reinterpret_cast<float*>(ws + L.S);
        f.rows = reinterpret_cast<float*>(ws + L.e);
        e = fact != nullptr ? sdm::launch_gdn_walk(1, f, fact, st) : sdm::launch_gdn_recur(s->dtype, 1, f, st);
    }
    r.state_in = dstate;
    r.y = dv;
    r.dy = dy;
    r.marks = reinterpret_cast<float*>(ws + L.dE);
    r.rows = reinterpret_cast<float*>(ws + L.d);
    r.state_out = dstate0;
    if (e == cudaSuccess) e = fact != nullptr ? sdm::launch_gdn_walk(2, r, fact, st) : sdm::launch_gdn_recur(s->dtype, 2, r, st);
    if (e == cudaSuccess && s->T > 0) {
        sdm::GdnGrads g{};
        g.a = f.a;
        g.dy = dy;
        g.S = f.marks; g.dE = r.marks; g.e = f.rows; g.d = r.rows;
        g.dq = dq; g.dk = dk; g.dalpha = dalpha; g.dbeta = dbeta;
        e = sdm::launch_gdn_grads(s->dtype, g, st);
    }
    return done(e, "sdm_gdn_backward");
}

size_t sdm_linear_workspace_bytes(const sdm_linear_shape* s) {
    if (linear_check(s) != SDM_OK) return 0;
    sdm::api_ok();
    return linear_fwd_ws(s);
}

size_t sdm_linear_backward_workspace_bytes(const sdm_linear_shape* s) {
    if (linear_check(s) != SDM_OK) return 0;
    sdm::api_ok();
    return s->M == 0 ? 0 : linear_bwd_layout(s).total;
}

sdm_status sdm_linear(const sdm_linear_shape* s, const void* x, const void* W, const float* bias, const void* residual,
                      void* out, void* pre, void* workspace, size_t workspace_bytes, sdm_stream_t stream) {
    SDM_TRY(linear_check(s));
    if (s->M == 0) return sdm::api_ok();
    const size_t mn = static_cast<size_t>(s->M) * s->N * 2, need = linear_fwd_ws(s);
    const Buf bufs[] = {{"x", x, static_cast<size_t>(s->M) * s->K * 2, 16, false, false},
                        {"W", W, static_cast<size_t>(s->N) * s->K * 2, 16, false, false},
                        {"bias", bias, static_cast<size_t>(s->N) * 4, 16, true, false},
                        {"residual", residual, mn, 16, true, false}, {"out", out, mn, 16, false, true},
                        {"pre", pre, mn, 16, true, true}, {"workspace", workspace, need, 16, true, true}};
    // residual == out is allowed: each element is read by the thread that overwrites it
    SDM_TRY(check_bufs("sdm_linear", bufs, 7, 3, 4));
    SDM_TRY(check_ws("sdm_linear", workspace, workspace_bytes, need));
    int* err = nullptr;
    SDM_TRY(sdm::api_status_word(&err));
    const sdm::LinearOut o{bias, residual, pre, out, s->act};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e = sdm::linear_skinny(s->M)
                        ? sdm::launch_linear_skinny(x, W, static_cast<int>(s->M), s->N, s->K, o, st)
                        : sdm::launch_linear(x, false, W, false, s->M, s->N, s->K, o, static_cast<float*>(workspace), err, st);
    return done(e, "sdm_linear");
}

sdm_status sdm_linear_backward(const sdm_linear_shape* s, const void* x, const void* W, const void* pre, const void* dout,
                               void* dx, void* dW, float* dbias, void* workspace, size_t workspace_bytes, sdm_stream_t stream) {
    SDM_TRY(linear_check(s));
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const size_t mn = static_cast<size_t>(s->M) * s->N * 2, mk = static_cast<size_t>(s->M) * s->K * 2,
                 nk = static_cast<size_t>(s->N) * s->K * 2;
    const LinearBwdLayout L = linear_bwd_layout(s);
    const size_t need = s->M == 0 ? 0 : L.total;
    const Buf bufs[] = {{"x", x, mk, 16, dW == nullptr, false}, {"W", W, nk, 16, dx == nullptr || s->M == 0, false},
                        {"pre", pre, mn, 16, s->act == SDM_ACT_NONE, false}, {"dout", dout, mn, 16, false, false},
                        {"dx", dx, mk, 16, true, true}, {"dW", dW, nk, 16, true, true},
                        {"dbias", dbias, static_cast<size_t>(s->N) * 4, 16, true, true},
                        {"workspace", workspace, need, 16, true, true}};
    SDM_TRY(check_bufs("sdm_linear_backward", bufs, 8));
    SDM_TRY(check_ws("sdm_linear_backward", workspace, workspace_bytes, need));
    cudaError_t e = cudaSuccess;
    if (s->M == 0) {
        if (dW != nullptr) e = cudaMemsetAsync(dW, 0, nk, st);
        if (e == cudaSuccess && dbias != nullptr) e = cudaMemsetAsync(dbias, 0, static_cast<size_t>(s->N) * 4, st);
        return done(e, "sdm_linear_backward");
    }
    int* err = nullptr;
    SDM_TRY(sdm::api_status_word(&err));
    char* ws = static_cast<char*>(workspace);
    const bool products = dx != nullptr || dW != nullptr, keep = products && s->act != SDM_ACT_NONE;
    void* dp = keep ? ws + L.dp : nullptr;
    if (keep || dbias != nullptr)
        e = sdm::launch_linear_dact(dout, pre, s->act, s->M, s->N, dp, dbias, reinterpret_cast<float*>(ws + L.part), st);
    const void* g = keep ? dp : dout;
    float* split = reinterpret_cast<float*>(ws + L.split);
    if (e == cudaSuccess && dx != nullptr)
        e = sdm::launch_linear(g, false, W, true, s->M, s->K, s->N, sdm::LinearOut{nullptr, nullptr, nullptr, dx, SDM_ACT_NONE}, split, err, st);
    if (e == cudaSuccess && dW != nullptr)
        e = sdm::launch_linear(g, true, x, true, s->N, s->K, s->M, sdm::LinearOut{nullptr, nullptr, nullptr, dW, SDM_ACT_NONE}, split, err, st);
    return done(e, "sdm_linear_backward");
}

}  // extern "C"
