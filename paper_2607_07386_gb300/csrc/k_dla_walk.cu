// Linear attention with a decay per head, in fp32: the walk in chunks of 32 tokens, and the single token.
//
// Within a chunk of n tokens (walked forwards, i and j from 0)
//   o_i = inter lam^(i+1) S^T r_i + intra sum_{j <= i} lam^(i-j) (r_i.k_j) v_j
//   S  <- lam^n S + add sum_j lam^(n-1-j) k_j v_j^T
// and, walked backwards from the last token, o_i takes lam^(n-1-i) S and j >= i, S takes lam^(j+1).  No power of
// the decay is above 1 for log_decay <= 0, so nothing can overflow however fast a head forgets.
//
// A CTA takes 32 columns of one state: the state lies in registers and, for the reads, in shared memory;
// r, k and v of the next chunk are on their way while this one is computed.  Every CTA of a chain takes the whole of P for itself: with
// d_v = 128 four times.  Bound by the fp32 units' and shared memory's latencies, which two CTAs an SM hide of each other (128 registers
// a thread to widths of 128; 252 at 256 in float32, and one CTA); 256 threads were faster than 128 or 512.  4 x 8 heads of 64 x 1,024
// tokens, forward: 91 us; 8 x 16 heads of 128 x 1,024: 601, and 1,656 backward; the odd backward of 3 x 6 heads of 64 x 96, up to 333
// tokens: 68 us, with float32 sums throughout.
//
// The single token reads and writes its state once, eight rows of four columns a thread, all its loads in flight together, and is bound by memory:
// 256 sequences, 16 heads of 128 x 128 (537 MB): 84.5 us, 0.94 of the copy bandwidth; one sequence: 5.9 us, a launch.
#include "dla_internal.h"
#include "sdm_common.cuh"

namespace sdm {

namespace {

constexpr int C = DLA_C32, WT = 256, COLS = 32;

template <int DA>
struct WalkSmem {
    float r[C][DA + 4], k[C][DA + 4], S[COLS][DA + 4];       // S transposed; rows four banks apart
    float v[COLS][C + 4], gv[C][COLS + 4], P[C][C + 4];      // v transposed; v times its weight in the state
    float pw[C + 1], lam[2][2];                              // lam^n; of a whole and of the partial chunk in two parts
};

template <class D>
__device__ __forceinline__ const uint4* token_ptr(const void* base, int64_t at) {
    return reinterpret_cast<const uint4*>(static_cast<const typename D::T*>(base) + at);
}
template <class D>
__device__ __forceinline__ void put_pair(void* out, int64_t at, float a, float b);
template <> __device__ __forceinline__ void put_pair<F32>(void* out, int64_t at, float a, float b) {
    *reinterpret_cast<float2*>(static_cast<float*>(out) + at) = make_float2(a, b);
}
template <> __device__ __forceinline__ void put_pair<BF16>(void* out, int64_t at, float a, float b) {
    *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(out) + at) = __floats2bfloat162_rn(a, b);
}

template <class D>
__device__ __forceinline__ void put_one(void* out, int64_t at, float x);
template <> __device__ __forceinline__ void put_one<F32>(void* out, int64_t at, float x) { static_cast<float*>(out)[at] = x; }
template <> __device__ __forceinline__ void put_one<BF16>(void* out, int64_t at, float x) { static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(x); }

template <class D, int DA, bool SUMS>
__global__ void __launch_bounds__(WT) k_dla_walk(const DlaWalk w) {
    extern __shared__ __align__(16) unsigned char raw[];
    WalkSmem<DA>& sm = *reinterpret_cast<WalkSmem<DA>*>(raw);
    const int tid = threadIdx.x;
    const int nseg = SUMS ? w.segs - 1 : w.segs;
    const int seg = blockIdx.x % nseg;
    int slice = blockIdx.x / nseg, role = 0;
    while (slice >= w.slices[role]) slice -= w.slices[role++];
    const DlaRole& ro = w.role[role];
    const int b = blockIdx.z, h = blockIdx.y, col0 = slice * COLS;
    const int len = dla_length(w, b);
    const int da = ro.da, db = ro.db;
    const int64_t chain = static_cast<int64_t>(b) * w.H + h;
    const float ld = __ldg(w.log_decay + h);
    const int chunks = (len + C - 1) / C;
    const int c0 = min(seg * w.seg_chunks, chunks), c1 = seg == w.segs - 1 ? chunks : min(c0 + w.seg_chunks, chunks);
    auto chunk_at = [&](int c) { return ro.reverse ? chunks - 1 - c : c; };
    auto tokens_in = [&](int c) { return min(C, len - chunk_at(c) * C); };

    const int hr = h / (w.H / ro.hr), hk = h / (w.H / ro.hk), hv = h / (w.H / ro.hv);
    const int64_t rb = gdn_base(w.token_major, b, hr, ro.hr, w.T, da), rs = gdn_stride(w.token_major, ro.hr, da);
    const int64_t kb = gdn_base(w.token_major, b, hk, ro.hk, w.T, da), ks = gdn_stride(w.token_major, ro.hk, da);
    const int64_t vb = gdn_base(w.token_major, b, hv, ro.hv, w.T, db), vs = gdn_stride(w.token_major, ro.hv, db);

    // pieces of 16 bytes: PR per row of r and k, NR of them a thread
    constexpr int PR = DA / D::E, NR = C * PR / WT, PV = COLS / D::E;
    uint4 ru[NR > 0 ? NR : 1], ku[NR > 0 ? NR : 1], vu;
    auto fetch = [&](int c) {
        const int t0 = chunk_at(c) * C, n = tokens_in(c);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = tid + i * WT, row = p / PR, x = p % PR * D::E;
            const bool on = row < n && x < da;
            if (!SUMS) ru[i] = on ? __ldg(token_ptr<D>(ro.r, rb + (t0 + row) * rs + x)) : make_uint4(0, 0, 0, 0);
            ku[i] = on ? __ldg(token_ptr<D>(ro.k, kb + (t0 + row) * ks + x)) : make_uint4(0, 0, 0, 0);
        }
        const int row = tid / PV, x = col0 + tid % PV * D::E;
        vu = row < n && x < db ? __ldg(token_ptr<D>(ro.v, vb + (t0 + row) * vs + x)) : make_uint4(0, 0, 0, 0);
    };
    auto put = [&](int n) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = tid + i * WT, row = p / PR, x = p % PR * D::E;
            float f[8];
            if (!SUMS) {
                unpack16<D>(ru[i], f);
#pragma unroll
                for (int e = 0; e < D::E; e += 4) *reinterpret_cast<float4*>(&sm.r[row][x + e]) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
            }
            unpack16<D>(ku[i], f);
#pragma unroll
            for (int e = 0; e < D::E; e += 4) *reinterpret_cast<float4*>(&sm.k[row][x + e]) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
        }
        const int row = tid / PV, x = tid % PV * D::E;
        if (row < C) {
            float f[8];
            unpack16<D>(vu, f);
            const float g = row < n ? ro.add * (ro.reverse ? sm.pw[row + 1] : sm.pw[n - 1 - row]) : 0.f;
#pragma unroll
            for (int e = 0; e < D::E; ++e) sm.v[x + e][row] = f[e];
#pragma unroll
            for (int e = 0; e < D::E; e += 4) *reinterpret_cast<float4*>(&sm.gv[row][x + e]) = make_float4(g * f[e], g * f[e + 1], g * f[e + 2], g * f[e + 3]);
        }
    };

    if (c0 < c1) fetch(c0);
    if (tid <= C) sm.pw[tid] = dla_pow(ld, tid);             // read after the loop's first barrier
    if (tid >= 64 && tid < 66) {
        const float2 f = dla_pow2(ld, tid == 64 ? C : len - (chunks - 1) * C);
        sm.lam[tid - 64][0] = f.x;
        sm.lam[tid - 64][1] = f.y;
    }
    if (SUMS && seg == 0 && col0 == 0 && tid >= 96 && tid < 99) dla_piece_pow(w, role, chain, ld, len, C, tid - 96);
    // This thread's part of the state: R rows x 4 columns.
    constexpr int R = DA / 32;
    const int cg = (tid & 7) * 4, x0 = (tid >> 3) * R;
    float S[R][4];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i][e] = 0.f;
    const int64_t per = static_cast<int64_t>(da) * db;
    auto at = [&](int x, int c) { return ro.transposed ? static_cast<int64_t>(col0 + c) * da + x : static_cast<int64_t>(x) * db + col0 + c; };
    // Pieces: [0] is the first state, [s + 1] what segment s adds, and for the second launch the state after it.
    float* const pieces = w.seg_state + w.seg_role[role] + chain * w.segs * per;
    if (!SUMS || seg == 0) {
        const float* const from = !SUMS && w.segs > 1 ? pieces + seg * per : ro.state_in == nullptr ? nullptr : ro.state_in + chain * per;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool on = x0 + i < da && col0 + cg + e < db;
                if (on && from != nullptr) S[i][e] = from[at(x0 + i, cg + e)];
                if (SUMS) {
                    if (on) pieces[at(x0 + i, cg + e)] = S[i][e];
                    S[i][e] = 0.f;
                }
            }
    }

    // Outputs: rows ti and ti + 1, columns tc and tc + 16 (rows of k, S and v that lie in different banks), of P alike.
    const int ti = (tid >> 4) * 2, tc = tid & 15;
    for (int c = c0; c < c1; ++c) {
        const int t0 = chunk_at(c) * C, n = tokens_in(c);
        __syncthreads();
        put(n);
        if (!SUMS) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < R; i += 2)               // rows past da stay zero, whatever k holds of them
                    *reinterpret_cast<float2*>(&sm.S[cg + e][x0 + i]) = x0 + i < da ? make_float2(S[i][e], S[i + 1][e]) : make_float2(0.f, 0.f);
        }
        __syncthreads();
        if (c + 1 < c1) fetch(c + 1);
        if (!SUMS) {
            float2 p[2][2], o[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) p[i][j] = o[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int x = 0; x < da; x += 4) {                // da is a multiple of 4
                float4 r[2], k[2], s[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    r[i] = *reinterpret_cast<const float4*>(&sm.r[ti + i][x]);
                    k[i] = *reinterpret_cast<const float4*>(&sm.k[tc + 16 * i][x]);
                    s[i] = *reinterpret_cast<const float4*>(&sm.S[tc + 16 * i][x]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        p[i][j] = __ffma2_rn(make_float2(r[i].x, r[i].y), make_float2(k[j].x, k[j].y), p[i][j]);
                        p[i][j] = __ffma2_rn(make_float2(r[i].z, r[i].w), make_float2(k[j].z, k[j].w), p[i][j]);
                        o[i][j] = __ffma2_rn(make_float2(r[i].x, r[i].y), make_float2(s[j].x, s[j].y), o[i][j]);
                        o[i][j] = __ffma2_rn(make_float2(r[i].z, r[i].w), make_float2(s[j].z, s[j].w), o[i][j]);
                    }
            }
            float y[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = ti + i;
                const float f = ro.inter * (ro.reverse ? sm.pw[max(n - 1 - row, 0)] : sm.pw[row + 1]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = tc + 16 * j, far = ro.reverse ? col - row : row - col;
                    sm.P[row][col] = far >= 0 ? ro.intra * sm.pw[far >= 0 ? far : 0] * (p[i][j].x + p[i][j].y) : 0.f;
                    y[i][j] = f * (o[i][j].x + o[i][j].y);
                }
            }
            __syncthreads();
            float2 z[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) z[i][j] = make_float2(y[i][j], 0.f);
#pragma unroll 4
            for (int j = 0; j < C; j += 4) {
                float4 q[2], v[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    q[i] = *reinterpret_cast<const float4*>(&sm.P[ti + i][j]);
                    v[i] = *reinterpret_cast<const float4*>(&sm.v[tc + 16 * i][j]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        z[i][e] = __ffma2_rn(make_float2(q[i].x, q[i].y), make_float2(v[e].x, v[e].y), z[i][e]);
                        z[i][e] = __ffma2_rn(make_float2(q[i].z, q[i].w), make_float2(v[e].z, v[e].w), z[i][e]);
                    }
            }
            // A token past this one in the walk counts with a zero, but not where its v is not finite; one past the length does too,
            // but not where its power is infinite (of states that grow).  Then it is left out by a test (tests in the loop above took
            // it from 1 to 4.7 thousand cycles).
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float sum = z[i][j].x + z[i][j].y;
                    if (gdn_finite(sum)) {
                        y[i][j] = sum;
                        continue;
                    }
                    float2 u = make_float2(y[i][j], 0.f);    // in the same order
#pragma unroll 1
                    for (int t = 0; t < n; t += 2) {
                        if (ro.reverse ? t >= ti + i : t <= ti + i) u.x = fmaf(sm.P[ti + i][t], sm.v[tc + 16 * j][t], u.x);
                        if (ro.reverse ? t + 1 >= ti + i && t + 1 < n : t + 1 <= ti + i) u.y = fmaf(sm.P[ti + i][t + 1], sm.v[tc + 16 * j][t + 1], u.y);
                    }
                    y[i][j] = u.x + u.y;
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (ti + i >= n) continue;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = col0 + tc + 16 * j;
                    if (col >= db) continue;
                    if (ro.partial) static_cast<float*>(ro.out)[(chain * w.T + t0 + ti + i) * db + col] = y[i][j];
                    else put_one<D>(ro.out, gdn_base(w.token_major, b, h, w.H, w.T, db) + (t0 + ti + i) * gdn_stride(w.token_major, w.H, db) + col, y[i][j]);
                }
            }
        }
        const float hi = sm.lam[n < C][0], lo = sm.lam[n < C][1];
        float add[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) add[i][e] = lo * S[i][e];
#pragma unroll 4
        for (int j = 0; j < (x0 < da ? n : 0); ++j) {
            const float4 v = *reinterpret_cast<const float4*>(&sm.gv[j][cg]);
            float k[R];
#pragma unroll
            for (int i = 0; i < R; i += 2) {
                const float2 a = *reinterpret_cast<const float2*>(&sm.k[j][x0 + i]);
                k[i] = a.x; k[i + 1] = a.y;
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                add[i][0] = fmaf(k[i], v.x, add[i][0]); add[i][1] = fmaf(k[i], v.y, add[i][1]);
                add[i][2] = fmaf(k[i], v.z, add[i][2]); add[i][3] = fmaf(k[i], v.w, add[i][3]);
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[i][e] = fmaf(hi, S[i][e], add[i][e]);
    }
    float* out = SUMS ? pieces + (seg + 1) * per : ro.state_out != nullptr ? ro.state_out + chain * per : nullptr;
    if (out != nullptr && (SUMS || seg == w.segs - 1)) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (x0 + i < da && col0 + cg + e < db) out[at(x0 + i, cg + e)] = S[i][e];
    }
    if (!SUMS) dla_zero_tail<D>(w, ro, b, h, col0, db - col0 < COLS ? db - col0 : COLS, len, seg, tid, WT);
}

template <class D, int DA, bool SUMS>
cudaError_t walk(const DlaWalk& w, cudaStream_t stream) {
    constexpr size_t smem = sizeof(WalkSmem<DA>);
    static std::atomic<unsigned long long> seen;
    cudaError_t e = allow_smem(k_dla_walk<D, DA, SUMS>, smem, seen);
    if (e != cudaSuccess) return e;
    int n = 0;
    for (int i = 0; i < w.roles; ++i) n += w.slices[i];
    const unsigned segs = static_cast<unsigned>(SUMS ? w.segs - 1 : w.segs);
    k_dla_walk<D, DA, SUMS><<<dim3(n * segs, w.H, w.B), WT, smem, stream>>>(w);
    return cudaGetLastError();
}
template <class D, int DA>
cudaError_t walks(const DlaWalk& w, cudaStream_t stream) {
    if (w.segs > 1) {
        cudaError_t e = walk<D, DA, true>(w, stream);
        if (e == cudaSuccess) e = launch_dla_prefix(w, C, stream);
        if (e != cudaSuccess) return e;
    }
    return walk<D, DA, false>(w, stream);
}
template <class D>
cudaError_t walk_width(DlaWalk& w, cudaStream_t stream) {
    int da = 0;
    for (int i = 0; i < w.roles; ++i) {
        da = w.role[i].da > da ? w.role[i].da : da;
        w.slices[i] = (w.role[i].db + COLS - 1) / COLS;
    }
    return da <= 64 ? walks<D, 64>(w, stream) : da <= 128 ? walks<D, 128>(w, stream) : walks<D, 256>(w, stream);
}

// The states at the starts of the pieces from what the pieces add; four values a thread.  The decay over a piece is multiplied on once
// for every piece after it, so it comes in two parts as in the walks (one chain of 152 pieces and a slow decay, state's error: 2.3e-6 in
// one part, 2e-7 in two); the first pass has taken it, for an exponential in 64 bits would take this kernel 2 us.
__global__ void __launch_bounds__(256) k_dla_prefix(const DlaWalk w, int C) {
    const int role = blockIdx.z % w.roles, b = blockIdx.z / w.roles, h = blockIdx.y;
    const DlaRole& ro = w.role[role];
    const int per = ro.width * ro.db, i = (blockIdx.x * 256 + threadIdx.x) * 4;      // a multiple of 16
    if (i >= per || ro.x0 != 0) return;                      // a role's pieces have one state
    const int chunks = (dla_length(w, b) + C - 1) / C, last = max(0, (chunks - 1) / w.seg_chunks);
    const int64_t chain = static_cast<int64_t>(b) * w.H + h;
    const float2* const pw = w.seg_pow + (role * static_cast<int64_t>(w.B) * w.H + chain) * 3;
    const float2 whole = pw[0], first = pw[1], end = pw[2];
    float4* p = reinterpret_cast<float4*>(w.seg_state + w.seg_role[role] + chain * w.segs * per + i);
    float4 S = *p;
    for (int s = 0; s + 1 < w.segs; ++s) {
        p += per / 4;
        if (s * w.seg_chunks < chunks) {                     // else it has no tokens, and adds nothing
            const float4 add = *p;
            const float2 f = s == last ? end : s == 0 ? first : whole;
            S.x = fmaf(f.x, S.x, fmaf(f.y, S.x, add.x)); S.y = fmaf(f.x, S.y, fmaf(f.y, S.y, add.y));
            S.z = fmaf(f.x, S.z, fmaf(f.y, S.z, add.z)); S.w = fmaf(f.x, S.w, fmaf(f.y, S.w, add.w));
        }
        *p = S;
    }
}

// Sums of shares, rounded once; four values a thread.
template <class D>
__global__ void __launch_bounds__(256) k_dla_join(const DlaSums sums, int B, int T, int token_major) {
    const DlaSum& j = sums.s[blockIdx.y];
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4, total = static_cast<int64_t>(B) * j.heads * T * j.d;
    if (i >= total) return;
    const int x = static_cast<int>(i % j.d);
    const int64_t row = i / j.d;
    const int t = static_cast<int>(row % T), h = static_cast<int>(row / T % j.heads), b = static_cast<int>(row / T / j.heads);
    const int64_t head = static_cast<int64_t>(T) * j.d, piece = static_cast<int64_t>(B) * j.heads * j.group * head;
    const float* part = j.part + (static_cast<int64_t>(b) * j.heads + h) * j.group * head + static_cast<int64_t>(t) * j.d + x;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < j.pieces; ++p)
        for (int g = 0; g < j.group; ++g) {
            const float4 f = __ldcs(reinterpret_cast<const float4*>(part + p * piece + g * head));
            s.x += f.x; s.y += f.y; s.z += f.z; s.w += f.w;
        }
    const int64_t at = gdn_base(token_major, b, h, j.heads, T, j.d) + t * gdn_stride(token_major, j.heads, j.d) + x;
    put_pair<D>(j.out, at, s.x, s.y);
    put_pair<D>(j.out, at + 2, s.z, s.w);
}

// One token: the state's two trips through HBM are all that counts.  A CTA takes 32 columns of one state, a warp 32 rows
// of them, a lane 8 rows x 4 columns, all in flight at once.
template <class D>
__device__ __forceinline__ void load_8(const void* base, int64_t at, int left, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += D::E) {
        const uint4 u = left > i ? __ldg(token_ptr<D>(base, at + i)) : make_uint4(0, 0, 0, 0);
        unpack16<D>(u, f + i);
    }
}
template <class D>
__global__ void __launch_bounds__(256) k_dla_step(const DlaStep r) {
    __shared__ __align__(16) float sh[8][32];
    const int b = blockIdx.z, h = blockIdx.y, hk = h / (r.H / r.Hk);
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const int row0 = 32 * warp + 8 * (lane >> 3), col = 32 * blockIdx.x + 4 * (lane & 7);
    const bool live = col < r.dv;                                // d_v is a multiple of 4
    int64_t slot = b;
    bool skip = false;
    if (r.slots != nullptr) {
        slot = __ldg(r.slots + b);
        if (slot >= r.n_slots && threadIdx.x == 0) flag_error(r.err, ERR_BAD_INDEX);
        skip = slot < 0 || slot >= r.n_slots;
    }
    const int64_t chain = static_cast<int64_t>(b) * r.H + h, kb = (static_cast<int64_t>(b) * r.Hk + hk) * r.dk;
    float* const st = r.state + (slot * r.H + h) * r.dk * r.dv + col;
    const int left = r.dk - row0;
    float4 S[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        S[i] = !skip && live && i < left ? __ldcs(reinterpret_cast<const float4*>(st + static_cast<int64_t>(row0 + i) * r.dv)) : make_float4(0.f, 0.f, 0.f, 0.f);
    float k[8], q[8], v[4] = {0.f, 0.f, 0.f, 0.f};
    load_8<D>(r.k, kb + row0, left, k);
    load_8<D>(r.q, kb + row0, left, q);
    if (live) {
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = load_elem<D>(r.v, chain * r.dv + col + c);
    }
    const float lam = dla_pow(__ldg(r.log_decay + h), 1);
    float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        S[i].x = fmaf(k[i], v[0], lam * S[i].x); S[i].y = fmaf(k[i], v[1], lam * S[i].y);
        S[i].z = fmaf(k[i], v[2], lam * S[i].z); S[i].w = fmaf(k[i], v[3], lam * S[i].w);
        if (!skip && live && i < left) __stcs(reinterpret_cast<float4*>(st + static_cast<int64_t>(row0 + i) * r.dv), S[i]);
        if (i < left) {                                          // past d_k: zero times a v that is not finite
            o[0] = fmaf(q[i], S[i].x, o[0]); o[1] = fmaf(q[i], S[i].y, o[1]);
            o[2] = fmaf(q[i], S[i].z, o[2]); o[3] = fmaf(q[i], S[i].w, o[3]);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        o[c] += __shfl_xor_sync(0xffffffffu, o[c], 8);
        o[c] += __shfl_xor_sync(0xffffffffu, o[c], 16);
    }
    if (warps > 1) {
        float4* const at = reinterpret_cast<float4*>(&sh[0][4 * (lane & 7)]);
        if (lane < 8) at[warp * 8] = make_float4(o[0], o[1], o[2], o[3]);
        __syncthreads();
        if (warp == 0 && lane < 8) {
            o[0] = o[1] = o[2] = o[3] = 0.f;
            for (int w = 0; w < warps; ++w) {
                const float4 p = at[w * 8];
                o[0] += p.x; o[1] += p.y; o[2] += p.z; o[3] += p.w;
            }
        }
    }
    if (warp == 0 && lane < 8 && live) {
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = skip ? 0.f : r.scale * o[c];
        put_pair<D>(r.y, chain * r.dv + col, o[0], o[1]);
        put_pair<D>(r.y, chain * r.dv + col + 2, o[2], o[3]);
    }
}

}  // namespace

void dla_plan(DlaWalk& w) {
    if (w.scan) {
        dla_scan_plan(w);
        return;
    }
    // The tokens are cut until there are three CTAs for every SM, one more than run at once; a piece keeps at least three
    // chunks, for the pass over the pieces' sums costs half of a walk and a launch.  One head of 64, 2,048 tokens: 318 us whole,
    // 41 cut; 4 x 8 heads, 1,024 tokens: 162 and 91.  Cut for one CTA an SM, for two and for three, forward (backward): 4 x 8 heads of 64 x
    // 1,024 99 (197), 78 (197), 90 (203); 8 heads of 128 x 2,048 136 (363), 118 (284), 133 (302); 3 x 6 heads of 64 x 96 x 333 47
    // (66), 46 (81), 46 (91), with the lengths of a ragged batch 47 (66), 43 (82), 43 (68).
    constexpr int64_t SMS = 152;
    int64_t ctas = 0;
    for (int i = 0; i < w.roles; ++i) ctas += (w.role[i].db + COLS - 1) / COLS;
    ctas *= static_cast<int64_t>(w.B) * w.H;
    const int64_t chunks = (w.T + C - 1) / C;
    int64_t segs = 3 * SMS / ctas;
    if (segs > chunks / 3) segs = chunks / 3;
    if (segs < 1) segs = 1;
    w.seg_chunks = static_cast<int>((chunks + segs - 1) / segs);
    w.segs = w.seg_chunks > 0 ? static_cast<int>((chunks + w.seg_chunks - 1) / w.seg_chunks) : 1;
}

cudaError_t launch_dla(int dtype, DlaWalk& w, cudaStream_t stream) {
    if (w.scan) return launch_dla_scan(w, stream);
    return dtype == SDM_F32 ? walk_width<F32>(w, stream) : walk_width<BF16>(w, stream);
}

cudaError_t launch_dla_prefix(const DlaWalk& w, int chunk, cudaStream_t stream) {
    int per = 0;
    for (int i = 0; i < w.roles; ++i) per = w.role[i].width * w.role[i].db > per ? w.role[i].width * w.role[i].db : per;
    k_dla_prefix<<<dim3((per / 4 + 255) / 256, w.H, w.B * w.roles), 256, 0, stream>>>(w, chunk);
    return cudaGetLastError();
}

cudaError_t launch_dla_join(int dtype, const DlaSums& sums, int B, int T, int token_major, cudaStream_t stream) {
    int64_t pieces = 0;
    for (int i = 0; i < sums.n; ++i) {
        const int64_t n = static_cast<int64_t>(B) * sums.s[i].heads * T * sums.s[i].d / 4;
        pieces = n > pieces ? n : pieces;
    }
    if (pieces == 0) return cudaSuccess;
    const dim3 grid(static_cast<unsigned>((pieces + 255) / 256), sums.n);
    if (dtype == SDM_F32) k_dla_join<F32><<<grid, 256, 0, stream>>>(sums, B, T, token_major);
    else k_dla_join<BF16><<<grid, 256, 0, stream>>>(sums, B, T, token_major);
    return cudaGetLastError();
}

cudaError_t launch_dla_step(int dtype, const DlaStep& s, cudaStream_t stream) {
    const dim3 grid((s.dv + 31) / 32, s.H, s.B);
    const int threads = 32 * ((s.dk + 31) / 32);
    if (dtype == SDM_F32) k_dla_step<F32><<<grid, threads, 0, stream>>>(s);
    else k_dla_step<BF16><<<grid, threads, 0, stream>>>(s);
    return cudaGetLastError();
}

}  // namespace sdm
