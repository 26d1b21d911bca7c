// C ABI of the decayed linear attention, the block norm and gradient clipping: argument checks, workspaces, launches.
// Declarations and semantics: include/sdm.h.
#include "api_check.h"
#include "dla_internal.h"

#include <algorithm>
#include <memory>
#include <new>

static_assert(sizeof(sdm_dla_shape) == 36, "sdm_dla_shape layout is part of the ABI");
static_assert(sizeof(sdm_block_norm_shape) == 32, "sdm_block_norm_shape layout is part of the ABI");
static_assert(sizeof(sdm_grad_tensor) == 32, "sdm_grad_tensor layout is part of the ABI");

namespace {

// ------------------------------------------------------------------ decayed linear attention
sdm_status dla_check(const sdm_dla_shape* s) {
    if (!s) return fail(SDM_ERR_INVALID_ARG, "shape is NULL");
    if (s->B < 0 || s->H < 0 || s->T < 0) return fail(SDM_ERR_INVALID_ARG, "B, H, T must be >= 0 (got %d, %d, %d)", s->B, s->H, s->T);
    if (s->B > 65535 || s->H > 65535) return fail(SDM_ERR_UNSUPPORTED, "B and H must be <= 65535 (got %d, %d)", s->B, s->H);
    if (s->T > INT_MAX - 64) return fail(SDM_ERR_UNSUPPORTED, "T too large (%d)", s->T);
    if (s->H > 0 && (s->H_k < 1 || s->H % s->H_k != 0))
        return fail(SDM_ERR_INVALID_ARG, "H must be a multiple of H_k >= 1 (got %d, %d)", s->H, s->H_k);
    if (s->dtype != SDM_F32 && s->dtype != SDM_BF16) return fail(SDM_ERR_INVALID_ARG, "unknown dtype %d", s->dtype);
    if (s->layout != SDM_HEAD_MAJOR && s->layout != SDM_TOKEN_MAJOR) return fail(SDM_ERR_INVALID_ARG, "unknown layout %d", s->layout);
    if (s->d_k < 1 || s->d_v < 1) return fail(SDM_ERR_INVALID_ARG, "d_k and d_v must be >= 1 (got %d, %d)", s->d_k, s->d_v);
    if (s->d_k > 256 || s->d_v > 256) return fail(SDM_ERR_UNSUPPORTED, "d_k and d_v must be <= 256 (got %d, %d)", s->d_k, s->d_v);
    const size_t es = esize(s->dtype);
    if (s->d_k * es % 16 != 0 || s->d_v * es % 16 != 0)
        return fail(SDM_ERR_UNSUPPORTED, "d_k and d_v times the element size must be multiples of 16 bytes (d_k=%d, d_v=%d)", s->d_k, s->d_v);
    if (static_cast<int64_t>(s->B) * s->H * s->T > (int64_t{1} << 31))
        return fail(SDM_ERR_UNSUPPORTED, "B * H * T must be at most 2^31 (got %d, %d, %d)", s->B, s->H, s->T);
    if (!(s->scale - s->scale == 0.f)) return fail(SDM_ERR_INVALID_ARG, "scale must be finite");
    return SDM_OK;
}

struct DlaSizes {
    size_t qk, v, state;
};
DlaSizes dla_sizes(const sdm_dla_shape* s) {
    const size_t es = esize(s->dtype), bt = static_cast<size_t>(s->B) * s->T;
    return DlaSizes{bt * s->H_k * s->d_k * es, bt * s->H * s->d_v * es, static_cast<size_t>(s->B) * s->H * s->d_k * s->d_v * 4};
}

sdm::DlaWalk dla_walk(const sdm_dla_shape* s, const float* log_decay, const int32_t* lengths, int roles) {
    sdm::DlaWalk w{};
    w.B = s->B; w.H = s->H; w.T = s->T;
    w.token_major = s->layout == SDM_TOKEN_MAJOR;
    w.log_decay = log_decay;
    w.lengths = lengths;
    w.roles = roles;
    return w;
}

// The roles of a call, the scan's with a wide contraction in two pieces, and where a workspace holds what: the pieces'
// states and decays, then the shares of the outputs that are sums (of value heads that share a key head, of the contraction's pieces).
struct DlaCall {
    const void* r; const void* k; const void* v;
    void* out;
    const float* state_in;
    float* state_out;
};
struct DlaLayout {
    sdm::DlaWalk w;
    sdm::DlaSums sums;
    int call[sdm::DLA_ROLES];     // the buffers that a role has, and the sum that it gives a share to (-1: none)
    int sum[sdm::DLA_ROLES];
    size_t share[sdm::DLA_ROLES], seg_pow, total;
};
DlaLayout dla_layout(const sdm_dla_shape* s, bool back) {
    DlaLayout L{};
    L.w = dla_walk(s, nullptr, nullptr, 0);
    const int H = s->H, Hk = s->H_k;
    const bool scan = sdm::dla_scan_pays(s->dtype, s->T, s->d_k, s->d_v);
    L.w.scan = scan;
    const size_t chains = static_cast<size_t>(s->B) * H;
    if (chains == 0) return L;                               // H_k may be anything then
    size_t floats = 0;
    size_t share[sdm::DLA_ROLES] = {};
    auto add = [&](int call, sdm::DlaRole r, int group) {
        const int cuts = scan && r.da > 128 ? 2 : 1;
        const bool sum = cuts * group > 1;
        r.width = r.da;
        r.partial = sum;
        const int job = sum ? L.sums.n++ : -1;
        if (sum) L.sums.s[job] = sdm::DlaSum{nullptr, nullptr, H / group, group, cuts, r.db};
        for (int c = 0; c < cuts; ++c) {
            const int i = L.w.roles++;
            L.w.role[i] = r;
            L.w.role[i].x0 = 128 * c;
            L.w.role[i].da = cuts == 1 ? r.width : c == 0 ? 128 : r.width - 128;
            L.call[i] = call;
            L.sum[i] = job;
            if (sum) {
                share[i] = floats;
                floats += chains * s->T * r.db;
            }
        }
    };
    sdm::DlaRole r{};
    if (!back) {
        r.hr = Hk; r.hk = Hk; r.hv = H; r.da = s->d_k; r.db = s->d_v;
        r.inter = r.intra = s->scale; r.add = 1.f;
        add(0, r, 1);
    } else {
        r.hr = H; r.hk = H; r.hv = Hk; r.da = s->d_v; r.db = s->d_k;                         // dq
        r.inter = r.intra = s->scale; r.add = 1.f; r.transposed = 1;
        add(0, r, H / Hk);
        r = sdm::DlaRole{};
        r.hr = Hk; r.hk = Hk; r.hv = H; r.da = s->d_k; r.db = s->d_v;                        // dv
        r.inter = 1.f; r.intra = r.add = s->scale; r.reverse = 1;
        add(1, r, 1);
        r = sdm::DlaRole{};
        r.hr = H; r.hk = H; r.hv = Hk; r.da = s->d_v; r.db = s->d_k;                         // dk
        r.inter = 1.f; r.intra = r.add = s->scale; r.reverse = 1; r.transposed = 1;
        add(2, r, H / Hk);
    }
    sdm::dla_plan(L.w);
    size_t state = 0;
    for (int i = 0; i < L.w.roles; ++i) {                    // a role's pieces have one state
        const sdm::DlaRole& q = L.w.role[i];
        L.w.seg_role[i] = q.x0 > 0 ? L.w.seg_role[i - 1] : static_cast<int64_t>(state);
        if (L.w.segs > 1 && q.x0 == 0) state += chains * L.w.segs * q.width * q.db;
    }
    L.seg_pow = state * 4;                                   // a state is a multiple of 16 floats
    const size_t pows = L.w.segs > 1 ? chains * L.w.roles * 3 * sizeof(float2) : 0;
    const size_t at = align256(L.w.span > 0 ? sdm::dla_scan_cut_bytes() : L.seg_pow + pows);
    for (int i = 0; i < L.w.roles; ++i) L.share[i] = at + share[i] * 4;
    L.total = at + align256(floats * 4);
    return L;
}
cudaError_t dla_run(int dtype, DlaLayout& L, const DlaCall* calls, char* ws, cudaStream_t stream) {
    L.w.seg_state = reinterpret_cast<float*>(ws);
    L.w.seg_pow = reinterpret_cast<float2*>(ws + L.seg_pow);
    for (int i = 0; i < L.w.roles; ++i) {
        sdm::DlaRole& r = L.w.role[i];
        const DlaCall& c = calls[L.call[i]];
        r.r = c.r; r.k = c.k; r.v = c.v;
        r.state_in = c.state_in;
        r.state_out = c.state_out;
        r.out = c.out;
        if (L.sum[i] < 0) continue;
        r.out = ws + L.share[i];
        sdm::DlaSum& s = L.sums.s[L.sum[i]];
        if (r.x0 == 0) s.part = reinterpret_cast<const float*>(r.out);
        s.out = c.out;
    }
    cudaError_t e = sdm::launch_dla(dtype, L.w, stream);
    if (e == cudaSuccess && L.sums.n > 0) e = sdm::launch_dla_join(dtype, L.sums, L.w.B, L.w.T, L.w.token_major, stream);
    return e;
}

// cut_polls > 0: as a test, with cut chains' states withheld and that limit to the waits for them.
sdm_status dla_forward(const char* who, const sdm_dla_shape* s, const void* q, const void* k, const void* v, const float* log_decay,
                       const int32_t* lengths, float* state, void* y, void* workspace, size_t workspace_bytes, int32_t cut_polls, sdm_stream_t stream) {
    const DlaSizes z = dla_sizes(s);
    DlaLayout L = dla_layout(s, false);
    const bool step = s->T == 1 && lengths == nullptr;       // on the kernel of sdm_dla_step, which takes no workspace
    const size_t need = step ? 0 : L.total;
    const Buf bufs[] = {{"q", q, z.qk, 16, false, false}, {"k", k, z.qk, 16, false, false}, {"v", v, z.v, 16, false, false},
                        {"log_decay", log_decay, static_cast<size_t>(s->H) * 4, 4, false, false},
                        {"lengths", lengths, static_cast<size_t>(s->B) * 4, 4, true, false},
                        {"state", state, z.state, 16, false, true}, {"y", y, z.v, 16, false, true},
                        {"workspace", workspace, need, 16, true, true}};
    SDM_TRY(check_bufs(who, bufs, 8));
    SDM_TRY(check_ws(who, workspace, workspace_bytes, need));
    SDM_TRY(sdm::api_status_word(&L.w.err));
    if (step) {
        const sdm::DlaStep d{q, k, v, log_decay, nullptr, state, y, s->B, s->H, s->H_k, s->d_k, s->d_v, s->B, s->scale, L.w.err};
        return done(sdm::launch_dla_step(s->dtype, d, reinterpret_cast<cudaStream_t>(stream)), who);
    }
    L.w.log_decay = log_decay;
    L.w.lengths = lengths;
    if (cut_polls > 0) {
        L.w.cut_polls = cut_polls;
        L.w.cut_hold = 1;
    }
    const DlaCall call{q, k, v, y, state, state};
    return done(dla_run(s->dtype, L, &call, static_cast<char*>(workspace), reinterpret_cast<cudaStream_t>(stream)), who);
}

// ------------------------------------------------------------------ block norm
sdm_status block_norm_check(const sdm_block_norm_shape* s) {
    if (!s) return fail(SDM_ERR_INVALID_ARG, "shape is NULL");
    if (s->M < 0 || s->D < 1 || s->gate_rows < 1)
        return fail(SDM_ERR_INVALID_ARG, "M must be >= 0, D and gate_rows >= 1 (got %lld, %d, %lld)", (long long)s->M, s->D, (long long)s->gate_rows);
    if (s->dtype != SDM_F32 && s->dtype != SDM_BF16) return fail(SDM_ERR_INVALID_ARG, "unknown dtype %d", s->dtype);
    if (s->D * esize(s->dtype) % 16 != 0) return fail(SDM_ERR_UNSUPPORTED, "D times the element size must be a multiple of 16 bytes (D=%d)", s->D);
    if (!sdm::block_norm_supported(s->D)) return fail(SDM_ERR_UNSUPPORTED, "D must be at most 16384 (got %d)", s->D);
    if (s->M > (int64_t{1} << 31)) return fail(SDM_ERR_UNSUPPORTED, "M must be at most 2^31 (got %lld)", (long long)s->M);
    if (!(s->eps >= 0.f && s->eps - s->eps == 0.f)) return fail(SDM_ERR_INVALID_ARG, "eps must be finite and >= 0");
    return SDM_OK;
}

// A gate for more rows than there are is one for all of them.
int64_t gate_rows(const sdm_block_norm_shape* s) { return std::max<int64_t>(1, std::min(s->gate_rows, s->M)); }

sdm_status with(const char* who, const char* name, const void* p, const char* other, bool there) {
    if (p != nullptr && !there) return fail(SDM_ERR_INVALID_ARG, "%s: %s without %s", who, name, other);
    return SDM_OK;
}

// ------------------------------------------------------------------ gradients
struct Range {
    uintptr_t from, to;
    int64_t tensor;           // -1: stats, -2: workspace
    bool written;
};
sdm_status grad_check(const char* who, int64_t n, const sdm_grad_tensor* t, bool clip) {
    if (n < 0) return fail(SDM_ERR_INVALID_ARG, "%s: n must be >= 0 (got %lld)", who, (long long)n);
    if (n > (1 << 24)) return fail(SDM_ERR_UNSUPPORTED, "%s: more than 2^24 tensors", who);
    if (n > 0 && t == nullptr) return fail(SDM_ERR_INVALID_ARG, "%s: tensors is NULL", who);
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        const sdm_grad_tensor& g = t[i];
        if (g.n < 0) return fail(SDM_ERR_INVALID_ARG, "%s: tensor %lld has n = %lld", who, (long long)i, (long long)g.n);
        if (g.n > (int64_t{1} << 40) || (total += g.n) > (int64_t{1} << 40)) return fail(SDM_ERR_UNSUPPORTED, "%s: more than 2^40 values", who);
        if ((g.dtype != SDM_F32 && g.dtype != SDM_BF16) || (clip && g.out_dtype != SDM_F32 && g.out_dtype != SDM_BF16))
            return fail(SDM_ERR_INVALID_ARG, "%s: unknown dtype of tensor %lld", who, (long long)i);
        if (g.n == 0) continue;
        if (g.grad == nullptr || (clip && g.out == nullptr)) return fail(SDM_ERR_INVALID_ARG, "%s: tensor %lld is NULL", who, (long long)i);
        if (reinterpret_cast<uintptr_t>(g.grad) % esize(g.dtype) != 0 || (clip && reinterpret_cast<uintptr_t>(g.out) % esize(g.out_dtype) != 0))
            return fail(SDM_ERR_INVALID_ARG, "%s: tensor %lld is not aligned to its values", who, (long long)i);
        if (clip && g.out == g.grad && g.out_dtype != g.dtype)
            return fail(SDM_ERR_INVALID_ARG, "%s: tensor %lld in place with another dtype", who, (long long)i);
    }
    return SDM_OK;
}
// Nothing written may overlap anything else.
sdm_status grad_overlaps(const char* who, int64_t n, const sdm_grad_tensor* t, bool clip, const float* stats, const void* ws, size_t ws_bytes) {
    constexpr int64_t FEW = 256;
    Range few[FEW];
    std::unique_ptr<Range[]> many;
    Range* r = few;
    if (2 * n + 2 > FEW) {
        many.reset(new (std::nothrow) Range[static_cast<size_t>(2 * n + 2)]);
        r = many.get();
        if (r == nullptr) return fail(SDM_ERR_UNSUPPORTED, "%s: no host memory for a list of %lld tensors", who, (long long)n);
    }
    int64_t m = 0;
    bool sorted = true;
    auto add = [&](const void* p, size_t bytes, int64_t tensor, bool written) {
        if (p == nullptr || bytes == 0) return;
        const uintptr_t x = reinterpret_cast<uintptr_t>(p);
        sorted = sorted && (m == 0 || r[m - 1].from <= x);
        r[m++] = Range{x, x + bytes, tensor, written};
    };
    for (int64_t i = 0; i < n; ++i) {
        const bool in_place = clip && t[i].out == t[i].grad;
        add(t[i].grad, static_cast<size_t>(t[i].n) * esize(t[i].dtype), i, in_place);
    }
    for (int64_t i = 0; clip && i < n; ++i)
        if (t[i].out != t[i].grad) add(t[i].out, static_cast<size_t>(t[i].n) * esize(t[i].out_dtype), i, true);
    add(stats, 8, -1, true);
    add(ws, ws_bytes, -2, true);
    if (!sorted) std::sort(r, r + m, [](const Range& a, const Range& b) { return a.from < b.from; });
    const Range *all = nullptr, *written = nullptr;          // of those before: the one that reaches furthest
    for (int64_t i = 0; i < m; ++i) {
        const Range* bad = r[i].written ? all : written;
        if (bad != nullptr && r[i].from < bad->to) {
            auto name = [&](const Range& x, char (&s)[48]) {
                if (x.tensor < 0) snprintf(s, sizeof(s), "%s", x.tensor == -1 ? "stats" : "the workspace");
                else snprintf(s, sizeof(s), "tensor %lld", (long long)x.tensor);
            };
            char a[48], b[48];
            name(*bad, a);
            name(r[i], b);
            return fail(SDM_ERR_INVALID_ARG, "%s: %s overlaps %s", who, a, b);
        }
        if (all == nullptr || r[i].to > all->to) all = r + i;
        if (r[i].written && (written == nullptr || r[i].to > written->to)) written = r + i;
    }
    return SDM_OK;
}

sdm_status grad_call(const char* who, int64_t n, const sdm_grad_tensor* t, bool clip, float max_norm, float* stats, void* ws, size_t ws_bytes,
                     sdm_stream_t stream) {
    SDM_TRY(grad_check(who, n, t, clip));
    if (!(max_norm >= 0.f)) return fail(SDM_ERR_INVALID_ARG, "%s: max_norm must be >= 0", who);
    if (stats == nullptr) return fail(SDM_ERR_INVALID_ARG, "%s: stats is NULL", who);
    if (reinterpret_cast<uintptr_t>(stats) % 4 != 0) return fail(SDM_ERR_INVALID_ARG, "%s: stats is not 4-byte aligned", who);
    const size_t need = align256(sdm::grad_bytes(n, t));
    SDM_TRY(check_ws(who, ws, ws_bytes, need));
    SDM_TRY(grad_overlaps(who, n, t, clip, stats, ws, need));
    return done(sdm::launch_grad(n, t, clip, max_norm, stats, ws, reinterpret_cast<cudaStream_t>(stream)), who);
}

}  // namespace

extern "C" {

size_t sdm_dla_workspace_bytes(const sdm_dla_shape* s) {
    if (dla_check(s) != SDM_OK) return 0;
    sdm::api_ok();
    return dla_layout(s, false).total;
}

size_t sdm_dla_backward_workspace_bytes(const sdm_dla_shape* s) {
    if (dla_check(s) != SDM_OK) return 0;
    sdm::api_ok();
    return dla_layout(s, true).total;
}

sdm_status sdm_dla_forward(const sdm_dla_shape* s, const void* q, const void* k, const void* v, const float* log_decay,
                           const int32_t* lengths, float* state, void* y, void* workspace, size_t workspace_bytes, sdm_stream_t stream) {
    SDM_TRY(dla_check(s));
    if (static_cast<size_t>(s->B) * s->H * s->T == 0) return sdm::api_ok();
    return dla_forward("sdm_dla_forward", s, q, k, v, log_decay, lengths, state, y, workspace, workspace_bytes, 0, stream);
}

sdm_status sdm_dla_plan(const sdm_dla_shape* s, int backward, int32_t* out, int n) {
    SDM_TRY(dla_check(s));
    if (!out || n < 0 || n > 4) return fail(SDM_ERR_INVALID_ARG, "sdm_dla_plan: out must be non-NULL and n in [0, 4]");
    const DlaLayout L = dla_layout(s, backward != 0);
    const int32_t v[4] = {L.w.scan, L.w.segs, L.w.seg_chunks, L.w.span > 0 ? sdm::dla_scan_cuts(L.w) : 0};
    for (int i = 0; i < n; ++i) out[i] = v[i];
    return sdm::api_ok();
}

sdm_status sdm_test_dla_wait_timeout(const sdm_dla_shape* s, const void* q, const void* k, const void* v, const float* log_decay,
                                     const int32_t* lengths, float* state, void* y, void* workspace, size_t workspace_bytes,
                                     int32_t wait_polls, sdm_stream_t stream) {
    const char* who = "sdm_test_dla_wait_timeout";
    SDM_TRY(dla_check(s));
    if (wait_polls < 1 || wait_polls > (1 << 24)) return fail(SDM_ERR_INVALID_ARG, "%s: wait_polls must be in [1, 2^24]", who);
    const DlaLayout L = dla_layout(s, false);
    if (L.w.span == 0 || sdm::dla_scan_cuts(L.w) == 0) return fail(SDM_ERR_UNSUPPORTED, "%s: no chain of this shape is cut", who);
    return dla_forward(who, s, q, k, v, log_decay, lengths, state, y, workspace, workspace_bytes, wait_polls, stream);
}

sdm_status sdm_dla_step(const sdm_dla_shape* s, const void* q, const void* k, const void* v, const float* log_decay, const int32_t* slots,
                        int32_t n_slots, float* state, void* y, sdm_stream_t stream) {
    SDM_TRY(dla_check(s));
    if (s->T != 1) return fail(SDM_ERR_INVALID_ARG, "sdm_dla_step needs shape->T == 1 (got %d)", s->T);
    if (n_slots < 0 || (slots == nullptr && n_slots < s->B))
        return fail(SDM_ERR_INVALID_ARG, "sdm_dla_step: n_slots = %d for B = %d sequences", n_slots, s->B);
    if (static_cast<size_t>(s->B) * s->H == 0) return sdm::api_ok();
    const DlaSizes z = dla_sizes(s);
    const Buf bufs[] = {{"q", q, z.qk, 16, false, false}, {"k", k, z.qk, 16, false, false}, {"v", v, z.v, 16, false, false},
                        {"log_decay", log_decay, static_cast<size_t>(s->H) * 4, 4, false, false},
                        {"slots", slots, static_cast<size_t>(s->B) * 4, 4, true, false},
                        {"state", state, static_cast<size_t>(n_slots) * s->H * s->d_k * s->d_v * 4, 16, false, true},
                        {"y", y, z.v, 16, false, true}};
    SDM_TRY(check_bufs("sdm_dla_step", bufs, 7));
    int* err = nullptr;
    SDM_TRY(sdm::api_status_word(&err));
    const sdm::DlaStep d{q, k, v, log_decay, slots, state, y, s->B, s->H, s->H_k, s->d_k, s->d_v, n_slots, s->scale, err};
    return done(sdm::launch_dla_step(s->dtype, d, reinterpret_cast<cudaStream_t>(stream)), "sdm_dla_step");
}

sdm_status sdm_dla_backward(const sdm_dla_shape* s, const void* q, const void* k, const void* v, const float* log_decay,
                            const int32_t* lengths, const float* state0, const void* dy, const float* dstate, void* dq, void* dk, void* dv,
                            float* dstate0, void* workspace, size_t workspace_bytes, sdm_stream_t stream) {
    SDM_TRY(dla_check(s));
    if (static_cast<size_t>(s->B) * s->H == 0) return sdm::api_ok();
    const DlaSizes z = dla_sizes(s);
    DlaLayout L = dla_layout(s, true);
    const Buf bufs[] = {{"q", q, z.qk, 16, false, false}, {"k", k, z.qk, 16, false, false}, {"v", v, z.v, 16, false, false},
                        {"log_decay", log_decay, static_cast<size_t>(s->H) * 4, 4, false, false},
                        {"lengths", lengths, static_cast<size_t>(s->B) * 4, 4, true, false},
                        {"state0", state0, z.state, 16, false, false}, {"dy", dy, z.v, 16, false, false},
                        {"dstate", dstate, z.state, 16, true, false}, {"dq", dq, z.qk, 16, false, true},
                        {"dk", dk, z.qk, 16, false, true}, {"dv", dv, z.v, 16, false, true},
                        {"dstate0", dstate0, z.state, 16, true, true}, {"workspace", workspace, L.total, 16, true, true}};
    SDM_TRY(check_bufs("sdm_dla_backward", bufs, 13));
    SDM_TRY(check_ws("sdm_dla_backward", workspace, workspace_bytes, L.total));
    SDM_TRY(sdm::api_status_word(&L.w.err));
    L.w.log_decay = log_decay;
    L.w.lengths = lengths;
    const DlaCall calls[] = {{dy, v, k, dq, state0, nullptr}, {k, q, dy, dv, dstate, dstate0}, {v, dy, q, dk, dstate, nullptr}};
    return done(dla_run(s->dtype, L, calls, static_cast<char*>(workspace), reinterpret_cast<cudaStream_t>(stream)), "sdm_dla_backward");
}

sdm_status sdm_block_norm(const sdm_block_norm_shape* s, const void* x, const void* y, const void* gate, const float* res_scale,
                          const float* gamma_post, const float* gamma_pre, void* h, void* z, sdm_stream_t stream) {
    const char* who = "sdm_block_norm";
    SDM_TRY(block_norm_check(s));
    SDM_TRY(with(who, "gate", gate, "y", y != nullptr));
    SDM_TRY(with(who, "res_scale", res_scale, "y", y != nullptr));
    SDM_TRY(with(who, "gamma_post", gamma_post, "y", y != nullptr));
    SDM_TRY(with(who, "h", h, "y", y != nullptr));
    SDM_TRY(with(who, "z", z, "gamma_pre", gamma_pre != nullptr));
    SDM_TRY(with(who, "gamma_pre", gamma_pre, "z", z != nullptr || s->M == 0));
    const size_t es = esize(s->dtype), rows = static_cast<size_t>(s->M) * s->D * es, v = static_cast<size_t>(s->D) * 4;
    const size_t gates = static_cast<size_t>((s->M + gate_rows(s) - 1) / gate_rows(s)) * s->D * es;
    if (s->M > 0 && y == nullptr && z == nullptr) return fail(SDM_ERR_INVALID_ARG, "%s: neither y nor z", who);
    const Buf bufs[] = {{"x", x, rows, 16, false, false}, {"y", y, rows, 16, true, false}, {"gate", gate, gates, 16, true, false},
                        {"res_scale", res_scale, v, 16, true, false}, {"gamma_post", gamma_post, v, 16, true, false},
                        {"gamma_pre", gamma_pre, v, 16, true, false}, {"h", h, rows, 16, y == nullptr, true}, {"z", z, rows, 16, true, true}};
    SDM_TRY(check_bufs(who, bufs, 8, 0, 6));                 // each row of x is read by the threads that write it to h
    if (s->M == 0) return sdm::api_ok();
    sdm::BlockNorm a{};
    a.M = s->M; a.gate_rows = gate_rows(s); a.D = s->D; a.eps = s->eps;
    a.x = x; a.y = y; a.gate = gate; a.res_scale = res_scale; a.gamma_post = gamma_post; a.gamma_pre = gamma_pre;
    a.h = h; a.z = z;
    return done(sdm::launch_block_norm(s->dtype, a, reinterpret_cast<cudaStream_t>(stream)), who);
}

size_t sdm_block_norm_backward_workspace_bytes(const sdm_block_norm_shape* s) {
    if (block_norm_check(s) != SDM_OK) return 0;
    sdm::api_ok();
    return align256(sdm::block_norm_backward_bytes(s->dtype, s->M, gate_rows(s), s->D));
}

sdm_status sdm_block_norm_backward(const sdm_block_norm_shape* s, const void* y, const void* h, const void* gate, const float* res_scale,
                                   const float* gamma_post, const float* gamma_pre, const void* dz, const void* dh, void* dx, void* dy,
                                   void* dgate, float* dres_scale, float* dgamma_post, float* dgamma_pre, void* workspace,
                                   size_t workspace_bytes, sdm_stream_t stream) {
    const char* who = "sdm_block_norm_backward";
    SDM_TRY(block_norm_check(s));
    const bool some = s->M > 0;
    SDM_TRY(with(who, "gate", gate, "y", y != nullptr || !some));
    SDM_TRY(with(who, "res_scale", res_scale, "y", y != nullptr || !some));
    SDM_TRY(with(who, "gamma_post", gamma_post, "y", y != nullptr || !some));
    SDM_TRY(with(who, "dy", dy, "y", y != nullptr || !some));
    SDM_TRY(with(who, "dgate", dgate, "gate", gate != nullptr || !some));
    SDM_TRY(with(who, "dres_scale", dres_scale, "res_scale", res_scale != nullptr));
    SDM_TRY(with(who, "dgamma_post", dgamma_post, "gamma_post", gamma_post != nullptr));
    SDM_TRY(with(who, "dgamma_pre", dgamma_pre, "gamma_pre", gamma_pre != nullptr));
    SDM_TRY(with(who, "dz", dz, "gamma_pre", gamma_pre != nullptr || !some));
    SDM_TRY(with(who, "gamma_pre", gamma_pre, "dz", dz != nullptr || !some));
    if (some && y == nullptr && dz == nullptr) return fail(SDM_ERR_INVALID_ARG, "%s: neither y nor dz", who);
    const size_t es = esize(s->dtype), rows = static_cast<size_t>(s->M) * s->D * es, v = static_cast<size_t>(s->D) * 4;
    const size_t gates = static_cast<size_t>((s->M + gate_rows(s) - 1) / gate_rows(s)) * s->D * es;
    const size_t need = align256(sdm::block_norm_backward_bytes(s->dtype, s->M, gate_rows(s), s->D));
    const Buf bufs[] = {{"y", y, rows, 16, true, false}, {"h", h, rows, 16, gamma_pre == nullptr, false}, {"gate", gate, gates, 16, true, false},
                        {"res_scale", res_scale, v, 16, true, false}, {"gamma_post", gamma_post, v, 16, true, false},
                        {"gamma_pre", gamma_pre, v, 16, true, false}, {"dz", dz, rows, 16, true, false}, {"dh", dh, rows, 16, true, false},
                        {"dx", dx, rows, 16, false, true}, {"dy", dy, rows, 16, y == nullptr, true}, {"dgate", dgate, gates, 16, true, true},
                        {"dres_scale", dres_scale, v, 16, true, true}, {"dgamma_post", dgamma_post, v, 16, true, true},
                        {"dgamma_pre", dgamma_pre, v, 16, true, true}, {"workspace", workspace, need, 16, true, true}};
    SDM_TRY(check_bufs(who, bufs, 15, 7, 8));                // each row of dh is read by the threads that write it to dx
    SDM_TRY(check_ws(who, workspace, workspace_bytes, need));
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (!some) {
        cudaError_t e = cudaSuccess;
        for (float* p : {dres_scale, dgamma_post, dgamma_pre})
            if (p != nullptr && e == cudaSuccess) e = cudaMemsetAsync(p, 0, v, st);
        return done(e, who);
    }
    sdm::BlockNorm a{};
    a.M = s->M; a.gate_rows = gate_rows(s); a.D = s->D; a.eps = s->eps;
    a.h = const_cast<void*>(h); a.y = y; a.gate = gate; a.res_scale = res_scale; a.gamma_post = gamma_post; a.gamma_pre = gamma_pre;
    a.dz = dz; a.dh = dh; a.dx = dx; a.dy = dy; a.dgate = dgate;
    a.dres_scale = dres_scale; a.dgamma_post = dgamma_post; a.dgamma_pre = dgamma_pre;
    a.ws = static_cast<float*>(workspace);
    return done(sdm::launch_block_norm_backward(s->dtype, a, st), who);
}

size_t sdm_grad_workspace_bytes(int64_t n, const sdm_grad_tensor* tensors) {
    if (grad_check("sdm_grad_workspace_bytes", n, tensors, false) != SDM_OK) return 0;
    sdm::api_ok();
    return align256(sdm::grad_bytes(n, tensors));
}

sdm_status sdm_grad_norm(int64_t n, const sdm_grad_tensor* tensors, float max_norm, float* stats, void* workspace, size_t workspace_bytes,
                         sdm_stream_t stream) {
    return grad_call("sdm_grad_norm", n, tensors, false, max_norm, stats, workspace, workspace_bytes, stream);
}

sdm_status sdm_grad_clip(int64_t n, const sdm_grad_tensor* tensors, float max_norm, float* stats, void* workspace, size_t workspace_bytes,
                         sdm_stream_t stream) {
    return grad_call("sdm_grad_clip", n, tensors, true, max_norm, stats, workspace, workspace_bytes, stream);
}

}  // extern "C"
