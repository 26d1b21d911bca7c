// Linear attention with a decay per head on the tensor cores: bf16, chunks of 64 tokens, widths of the contraction up to 128 (wider
// ones are cut in two, whose shares of the outputs are added up: P and what is read of S are sums over the width).
//
// A CTA walks one state, 128 columns of it (db), over its chunks; every product has 128 rows, TMEM lanes = columns of the state:
//   1  P[i, j]  = r_i.k_j                       A = [r; k] in shared memory (the k half is not used), B = k
//   2  I[c, i]  = sum_x S[x, c] r_i[x]          A = S transposed, two bf16 parts in TMEM
//   3  O[c, i]  = sum_j v_j[c] W_ij P_ij        A = v as TMA leaves it, B = the weighted P as two bf16 parts in shared memory
//   4  D[c, x]  = sum_j g_j v_j[c] k_j[x]       A = g v transposed, three bf16 parts in TMEM, B = k
// and out_i = w_i I + O, S <- lam^n S + D, in float32 and with lam^n in two parts.  W, w and g hold the powers of the decay
// (dla_internal.h).  r and k are used as TMA leaves them; v goes through registers, which transposes it, scales it and keeps
// what lies past the length out of the products.
//
// bf16 parts: g v has 8 + 24 significant bits, three parts keep 24 of them, so that the state is as good as a float32
// sum; S and the weighted P only reach outputs that are rounded to 2^-9, and two parts keep 16 bits, as they do for g v where
// no state is asked for.
//
// Only D goes from one chunk to the next, and it does not depend on S: six groups of warps work on different stages of
// neighbouring chunks, each handing over through mbarriers.
//
// Bound by that chain: a chunk takes 1.9 us, 3,650 cycles, of which 2,050 are its 56 MMAs (32 cycles each with A in TMEM, 48
// with A in shared memory) and most of the rest hand-overs, 250 cycles from a product's end to the warps that read it.
// 8 x 16 heads of 128 x 4,096 tokens: forward 135 us (64 chunks, and 13 us for the first and the last), 0.6 of the copy bandwidth (537
// MB of q, k, v and y are 79); backward, three runs of this walk, 384 chains spread over the SMs, 377 us (405 in three rounds of whole
// chains).  Tried and no faster, forward: P by products of 64 rows and lanes moved by 16 (136 to 162 us), three warps that issue (137), the
// state's product first (140), waits that sleep (148).
//
// A value of v that is not finite must stay out of the outputs before its token, which share its products: v is zero in
// them from that token on, its column's outputs from there are NaN, and so is the column of the state.
#include "dla_internal.h"
#include "gdn_tc.cuh"
#include "sdm_common.cuh"

#include <algorithm>
#include <climits>
#include <cstddef>

namespace sdm {

namespace {

using namespace gdn;

constexpr int SW = 8, VW = 8, OW = 4, PW = 4;  // warps: state, v, outputs, and (the last four) P, P, products, copies
constexpr int ST = 32 * (SW + VW + OW + PW);
constexpr int64_t SMS = 152;
constexpr int LAUNCH_REGS = 80, STATE_REGS = 104, V_REGS = 80, REST_REGS = 56;
static_assert(SW * STATE_REGS + VW * V_REGS + (OW + PW) * REST_REGS <= (SW + VW + OW + PW) * LAUNCH_REGS, "register split");

// TMEM columns: S, two parts; D, 64 rows of da at a time; g v, three parts; P; O; I.
constexpr uint32_t S_COL = 0, D_COL = 128, V_COL = 192, P_COL = 288, O_COL = 352, I_COL = 416, T_COLS = 512;
constexpr int CUT_LEAST = 4;                   // chunks of a piece
constexpr int SPREAD_SAVES = 9;                // chunks
constexpr int WP = 68;                         // floats of a row of W, so that rows start four banks apart

template <int DA>
struct ScanTile {
    static constexpr uint32_t RK = 0, V = DA / 64 * 16384, BYTES = V + 16384;        // [r; k] per 64 of da; v per 64 columns
    static constexpr int STAGES = DA == 128 ? 3 : 4;
    static constexpr uint32_t PS = BYTES * STAGES, OUT = PS + 4 * MAT, CTL = OUT + 16384;       // P's parts, of two chunks; outputs
};
// Barriers.  Completed by copies and MMAs: a stage's tile; P; D (per 64 rows of da); S's parts read; O, and with it I.  By
// warps: the parts of P (and P taken out); of g v; of S; D taken out; O and I taken out; what lies past the length is zero.
// By both: a stage is free.  And every product of the walk.
enum { B_FULL = 0, B_FREE = 4, B_P = 8, B_D, B_D1, B_SFREE, B_O, B_PS, B_V, B_S, B_DFREE, B_DFREE1, B_OFREE, B_ZERO, B_END, B_COUNT };
struct ScanCtl {
    float W[C * WP];
    float add[2][C], inter[2][C];              // weights of a whole chunk and of the partial one
    float pw[C + 1];
    float lam[2][2];                           // lam^n of both in two parts
    short first[4][2][128];                      // of a column: the chunk's first value (in the walk's order) that is not finite
    unsigned long long bar[B_COUNT];
    uint32_t tmem;
    int dead;
    int item[4];                               // of a list of chains that is cut: chain, first chunk, last, cut
};
template <int DA>
constexpr size_t scan_smem() { return 1024 + ScanTile<DA>::CTL + sizeof(ScanCtl); }
static_assert(scan_smem<128>() <= 227 * 1024 && scan_smem<64>() <= 227 * 1024, "shared memory");

struct ScanMaps {
    CUtensorMap r[DLA_ROLES], k[DLA_ROLES], v[DLA_ROLES], out[DLA_ROLES];
};

// Chains that are cut, in ascending order: the first `at` chunks of the walk are one piece, the rest another.  The first pieces come
// first, then the chains that are whole, then the rests, longest first.  A piece's place is drawn from a counter when it starts, so
// that a rest never waits for a piece that has not started (and hardly ever at all: whole chains lie between).  Where it has waited
// for w.cut_polls times about 0.1 us or more, it gives up, as every bounded wait: what it writes is undefined, and status bit 2 says so.
struct ScanCuts {
    int n;
    int chain[SMS], at[SMS];
    short order[SMS];                          // of the rests
};
constexpr int CUT_FLOATS = 128 * 128;          // a state that is handed over: up to 128 x 128, [x][column]
struct CutSpace {                              // at the start of the workspace
    unsigned next, ready[SMS];                 // zero at the launch
    alignas(256) float state[SMS][CUT_FLOATS];
};

// The next bf16 part of two floats, which keep what its rounding left: exact, in one mixed multiply-add each.
__device__ __forceinline__ uint32_t part2(float2& v) {
    const uint32_t u = pack2(v.x, v.y);
    asm("{\n .reg .b16 l, h, m;\n mov.b32 {l, h}, %2;\n mov.b16 m, 0xBF80;\n fma.rn.f32.bf16 %0, l, m, %0;\n fma.rn.f32.bf16 %1, h, m, %1;\n}\n"
        : "+f"(v.x), "+f"(v.y) : "r"(u));
    return u;
}
// A bf16 value of shared memory as a float.
__device__ __forceinline__ float load_bf16(const unsigned char* p) {
    float f;
    asm("{\n .reg .b16 h;\n mov.b16 h, %1;\n add.rn.f32.bf16 %0, h, 0f00000000;\n}\n" : "=f"(f) : "h"(*reinterpret_cast<const unsigned short*>(p)));
    return f;
}

template <int DA, bool SUMS>
__global__ void __launch_bounds__(ST, 1) k_dla_scan(const __grid_constant__ ScanMaps maps, const __grid_constant__ DlaWalk w, const __grid_constant__ ScanCuts cuts) {
    using L = ScanTile<DA>;
    extern __shared__ unsigned char raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t ring = (base + 1023u) & ~1023u;
    unsigned char* const ringp = raw + (ring - base);
    ScanCtl& ctl = *reinterpret_cast<ScanCtl*>(ringp + L::CTL);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool spread = !SUMS && w.span > 0;
    const int nseg = SUMS ? w.segs - 1 : w.segs, seg = spread ? 0 : blockIdx.x % nseg;
    int slice = blockIdx.x / nseg, role = 0, h = blockIdx.y, b = blockIdx.z, from = 0, to = INT_MAX, cut = -1;
    CutSpace* const space = reinterpret_cast<CutSpace*>(w.seg_state);
    if (spread) {
        int per = 0;
        for (int i = 0; i < w.roles; ++i) per += w.slices[i];
        if (tid == 0) {
            const int t = static_cast<int>(atomicAdd(&space->next, 1u)), total = per * w.H * w.B;
            int chain, j = -1, x = 0, y = INT_MAX;
            if (t < cuts.n) {
                j = t;
                chain = cuts.chain[j];
                y = cuts.at[j];
            } else if (t < total) {                          // the t - n'th whole one: j cut ones lie before it
                int lo = 0, hi = cuts.n;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (cuts.chain[mid] - mid <= t - cuts.n) lo = mid + 1;
                    else hi = mid;
                }
                chain = t - cuts.n + lo;
            } else {
                j = cuts.order[min(t - total, cuts.n - 1)];
                chain = cuts.chain[j];
                x = cuts.at[j];
            }
            ctl.item[0] = chain;
            ctl.item[1] = x;
            ctl.item[2] = y;
            ctl.item[3] = j;
        }
        __syncthreads();
        const int chain = ctl.item[0], bh = chain / per;
        slice = chain % per;
        h = bh % w.H;
        b = bh / w.H;
        from = ctl.item[1];
        to = ctl.item[2];
        cut = ctl.item[3];
    }
    while (slice >= w.slices[role]) slice -= w.slices[role++];
    const DlaRole& ro = w.role[role];
    const int col0 = slice * 128;
    const int len = dla_length(w, b), chunks = (len + C - 1) / C;
    const bool reverse = ro.reverse != 0;
    const int c0 = min(spread ? from : seg * w.seg_chunks, chunks);
    const int c1 = spread ? min(to, chunks) : seg == w.segs - 1 ? chunks : min(c0 + w.seg_chunks, chunks);
    const int todo = c1 - c0, outputs = SUMS ? 0 : todo, last_n = len - (chunks - 1) * C;       // tokens of the sequence's last chunk
    auto chunk_at = [&](int c) { return reverse ? chunks - 1 - (c0 + c) : c0 + c; };
    auto partial = [&](int c) { return chunk_at(c) == chunks - 1 && last_n < C; };
    const int64_t chain = static_cast<int64_t>(b) * w.H + h;
    const float ld = __ldg(w.log_decay + h);
    const int parts = ro.state_out != nullptr ? 3 : 2;       // of g v
    const uint32_t bars = smem_u32(&ctl.bar[0]);
    auto bar = [&](int i) { return bars + 8 * i; };
    if (tid == 0) {
        ctl.dead = 0;
        for (int i = 0; i < B_COUNT; ++i)
            mbar_init(bar(i), i >= B_FREE && i < B_P ? VW + 1 : i == B_PS ? 2 : i == B_V || i == B_ZERO ? VW : i == B_OFREE ? OW : i == B_S ? SW : i == B_DFREE || i == B_DFREE1 ? SW * 64 / DA : 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
    }
    if (warp == 0) tmem_alloc(smem_u32(&ctl.tmem), T_COLS);
    if (tid <= C) ctl.pw[tid] = dla_pow(ld, tid);
    if (tid >= 96 && tid < 98) {
        const int n = tid == 96 ? C : last_n;
        const float2 f = dla_pow2(ld, n);
        ctl.lam[tid - 96][0] = f.x;
        ctl.lam[tid - 96][1] = f.y;
    }
    if (SUMS && seg == 0 && col0 == 0 && tid >= 128 && tid < 131) dla_piece_pow(w, role, chain, ld, len, C, tid - 128);
    __syncthreads();
    if (tid < 2 * C) {
        const int k = tid / C, i = tid % C, n = k ? last_n : C;
        ctl.add[k][i] = i < n ? ro.add * (reverse ? ctl.pw[i + 1] : ctl.pw[n - 1 - i]) : 0.f;
        ctl.inter[k][i] = i < n ? ro.inter * (reverse ? ctl.pw[n - 1 - i] : ctl.pw[i + 1]) : 0.f;
    }
    if (!SUMS) {
        for (int p = tid; p < C * C; p += ST) {
            const int i = p / C, j = p % C, far = reverse ? j - i : i - j;
            ctl.W[i * WP + j] = far >= 0 ? ro.intra * ctl.pw[far] : 0.f;
        }
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = ctl.tmem;
    volatile int* dead = &ctl.dead;
    constexpr int SB = DA / 2;                               // TMEM columns of a part of S

    if (warp >= SW + VW + OW) {
        regs_dec<REST_REGS>();
        const int me = warp - (SW + VW + OW);
        if (me < 2) {                                        // P: row i of the chunk's tokens
            const int i = me * 32 + lane;
            const uint32_t lanes = tmem + (static_cast<uint32_t>(me * 32) << 16);
            const float* const wt = ctl.W + i * WP;
            unsigned char* const ps = ringp + L::PS;
            for (int c = 0; c < outputs; ++c) {
                await(bar(B_P), c & 1, dead);
                unsigned char* const to = ps + (c & 1) * 2 * MAT;
                const int n = partial(c) ? last_n : C;
                // A token past this one counts as zero, and where it is not finite, not as 0 times it: such products show in
                // `odd` (0 times each, added up), and are then left out by choice.  So are zeros past the length times a
                // power that is infinite (of states that grow).
                float2 odd = make_float2(0.f, 0.f);
                auto row = [&](int e, auto choose) {         // 32 columns
                    float p[32];
                    tmem_ld32(lanes + P_COL + 32 * e, p);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t u[4], l[4];
                        const float4 wa = *reinterpret_cast<const float4*>(wt + 32 * e + 8 * q), wb = *reinterpret_cast<const float4*>(wt + 32 * e + 8 * q + 4);
                        const float2 ww[4] = {make_float2(wa.x, wa.y), make_float2(wa.z, wa.w), make_float2(wb.x, wb.y), make_float2(wb.z, wb.w)};
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            float2 f = __fmul2_rn(ww[s], make_float2(p[8 * q + 2 * s], p[8 * q + 2 * s + 1]));
                            if (choose) {
                                const int j = 32 * e + 8 * q + 2 * s;
                                if (ww[s].x == 0.f || j >= n) f.x = 0.f;
                                if (ww[s].y == 0.f || j + 1 >= n) f.y = 0.f;
                            } else {
                                odd = __ffma2_rn(f, make_float2(0.f, 0.f), odd);
                            }
                            u[s] = part2(f);
                            l[s] = pack2(f.x, f.y);
                        }
                        unsigned char* const at = to + box_at(i, 4 * e + q);
                        *reinterpret_cast<uint4*>(at) = make_uint4(u[0], u[1], u[2], u[3]);
                        *reinterpret_cast<uint4*>(at + MAT) = make_uint4(l[0], l[1], l[2], l[3]);
                    }
                };
#pragma unroll 1
                for (int e = 0; e < 2; ++e) row(e, false);
                if (__any_sync(0xffffffffu, !(odd.x + odd.y == 0.f))) {
#pragma unroll 1
                    for (int e = 0; e < 2; ++e) row(e, true);
                }
                tc_before_sync();
                hand_over(bar(B_PS), lane);
            }
        } else if (me == 2) {                                // products, in an order that leaves every group of warps time
            const uint32_t id64 = mma_idesc(64);
            auto rk = [&](int c) {                           // 1
                const int s = c % L::STAGES;
                const uint32_t t = ring + s * L::BYTES;
                const uint64_t dr = sw128_desc(t + L::RK), dk = sw128_desc(t + L::RK + 8192);
                await(bar(B_FULL + s), (c / L::STAGES) & 1, dead);
                if (partial(c)) await(bar(B_ZERO), 0, dead);
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < DA / 16; ++kk)
                        mma_bf16(tmem + P_COL, dr + (kk / 4) * 1024 + (kk % 4) * 2, dk + (kk / 4) * 1024 + (kk % 4) * 2, id64, kk != 0);
                    mma_commit(bar(B_P));
                }
                __syncwarp();
            };
            if (!SUMS && todo > 0) rk(0);
            for (int c = 0; c < todo; ++c) {
                const int s = c % L::STAGES;
                const uint32_t t = ring + s * L::BYTES, ph = c & 1;
                const uint64_t dr = sw128_desc(t + L::RK), dkt = sw128_mn_desc(t + L::RK + 8192, 16384), dv = sw128_mn_desc(t + L::V, 8192),
                               dp = sw128_desc(ring + L::PS + (c & 1) * 2 * MAT);
                auto kv = [&](int x) {                       // 4, for 64 rows of da; lower parts first, here and below: their sums are small
                    if (elect_one()) {
#pragma unroll 1
                        for (int p = parts - 1; p >= 0; --p)
#pragma unroll
                            for (int kk = 0; kk < C / 16; ++kk)
                                mma_bf16_ta(tmem + D_COL, tmem + V_COL + p * 32 + kk * 8, dkt + x * 1024 + kk * 128, id64 | MN_B, p != parts - 1 || kk != 0);
                        mma_commit(bar(B_D + x));
                        if (SUMS && x == DA / 64 - 1) mma_commit(bar(B_FREE + s));
                    }
                    __syncwarp();
                };
                if (SUMS) await(bar(B_FULL + s), (c / L::STAGES) & 1, dead);
                await(bar(B_V), ph, dead);
                if (c > 0) await(bar(B_DFREE + DA / 64 - 1), (c - 1) & 1, dead);
                kv(0);
                if (!SUMS) {
                    await(bar(B_PS), ph, dead);
                    if (c + 1 < todo) rk(c + 1);
                }
                if (DA > 64) {
                    await(bar(B_DFREE), ph, dead);
                    kv(1);
                }
                if (SUMS) continue;
                await(bar(B_S), ph, dead);
                if (c > 0) await(bar(B_OFREE), (c - 1) & 1, dead);
                if (elect_one()) {                           // 2
#pragma unroll 1
                    for (int p = 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < DA / 16; ++kk)
                            mma_bf16_ta(tmem + I_COL, tmem + S_COL + p * SB + kk * 8, dr + (kk / 4) * 1024 + (kk % 4) * 2, id64, p != 1 || kk != 0);
                    mma_commit(bar(B_SFREE));
#pragma unroll 1
                    for (int p = 1; p >= 0; --p)             // 3
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16(tmem + O_COL, dv + kk * 128, dp + p * (MAT / 16) + kk * 2, id64 | MN_A, p != 1 || kk != 0);
                    mma_commit(bar(B_O));
                    mma_commit(bar(B_FREE + s));
                }
                __syncwarp();
            }
            if (todo > 0) {                                  // whatever became of the waits, no product outlives the CTA
                if (elect_one()) mma_commit(bar(B_END));
                __syncwarp();
                mbar_wait(bar(B_END), 0);
            }
        } else if (lane == 0) {                              // copies
            const int hr = h / (w.H / ro.hr), hk = h / (w.H / ro.hk), hv = h / (w.H / ro.hv);
            int loaded = 0;
            for (; loaded < todo; ++loaded) {
                const int s = loaded % L::STAGES;
                if (loaded >= L::STAGES) {
                    mbar_wait_or_dead(bar(B_FREE + s), (loaded / L::STAGES - 1) & 1, dead);
                    if (*dead) break;
                }
                const uint32_t t = ring + s * L::BYTES, fb = bar(B_FULL + s);
                const int at = chunk_at(loaded) * C;
                mbar_expect_tx(fb, SUMS ? L::BYTES - DA / 64 * 8192 : L::BYTES);
#pragma unroll
                for (int x = 0; x < DA / 64; ++x) {
                    tma_load_4d(t + L::RK + x * 16384 + 8192, &maps.k[role], ro.x0 + 64 * x, at, hk, b, fb);
                    if (!SUMS) tma_load_4d(t + L::RK + x * 16384, &maps.r[role], ro.x0 + 64 * x, at, hr, b, fb);
                }
                tma_load_4d(t + L::V, &maps.v[role], col0, at, hv, b, fb);
                tma_load_4d(t + L::V + 8192, &maps.v[role], col0 + 64, at, hv, b, fb);
            }
            for (int j = loaded > L::STAGES ? loaded - L::STAGES : 0; j < loaded; ++j)     // nor does a copy
                mbar_wait(bar(B_FULL + j % L::STAGES), (j / L::STAGES) & 1);
        }
    } else if (warp >= SW + VW) {                            // outputs: column `row`, all tokens
        regs_dec<REST_REGS>();
        const int quad = warp & 3, row = quad * 32 + lane, col = col0 + row;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const bool share = ro.partial != 0;
        float* const shares = static_cast<float*>(ro.out) + chain * w.T * ro.db + col;
        for (int c = 0; c < outputs; ++c) {
            const bool part = partial(c);
            const int n = part ? last_n : C, t0 = chunk_at(c) * C;
            unsigned char* const box = ringp + L::OUT;
            unsigned char* const yt = box + (row / 64) * 8192;
            const float* const wi = ctl.inter[part];
            if (!share) {                                    // the last copy has left the box
                if (warp == SW + VW && lane == 0) bulk_wait_read();
                asm volatile("bar.sync 1, %0;\n" ::"n"(32 * OW) : "memory");
            }
            await(bar(B_O), c & 1, dead);
            const int f0 = ctl.first[c & 3][0][row], f1 = ctl.first[c & 3][1][row], first = reverse ? max(f0, f1) : min(f0, f1);
            const bool odd = __any_sync(0xffffffffu, first != (reverse ? -1 : C));
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {                    // 16 tokens at a time
                float y[16], o[16];
                tmem_ld16_begin(lanes + I_COL + 16 * e, y);
                tmem_ld16_begin(lanes + O_COL + 16 * e, o);
                tmem_ld_wait(y);
                tmem_ld_wait(o);
                if (e == 3) {
                    tc_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(B_OFREE));
                }
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(wi + 16 * e + j);
                    const float2 a = __ffma2_rn(make_float2(f.x, f.y), make_float2(y[j], y[j + 1]), make_float2(o[j], o[j + 1]));
                    const float2 d = __ffma2_rn(make_float2(f.z, f.w), make_float2(y[j + 2], y[j + 3]), make_float2(o[j + 2], o[j + 3]));
                    y[j] = a.x; y[j + 1] = a.y; y[j + 2] = d.x; y[j + 3] = d.y;
                }
                if (odd || part) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int i = 16 * e + j;            // a column's outputs from its first odd value on
                        y[j] = i >= n ? 0.f : (reverse ? i <= first : i >= first) ? gdn_nan() : y[j];
                    }
                }
                if (share) {
                    if (col < ro.db) {
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (t0 + 16 * e + j < w.T) __stcs(shares + static_cast<int64_t>(t0 + 16 * e + j) * ro.db, y[j]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        const uint32_t u = pack2(y[j], y[j + 1]);
                        *reinterpret_cast<unsigned short*>(yt + sw128_at(16 * e + j, row % 64)) = static_cast<unsigned short>(u);
                        *reinterpret_cast<unsigned short*>(yt + sw128_at(16 * e + j + 1, row % 64)) = static_cast<unsigned short>(u >> 16);
                    }
                }
            }
            if (share) continue;
            fence_async();
            asm volatile("bar.sync 1, %0;\n" ::"n"(32 * OW) : "memory");
            if (warp == SW + VW && lane == 0) {
                const uint32_t src = smem_u32(box);
                if (!*dead) {
                    tma_store_4d(&maps.out[role], src, col0, t0, h, b);
                    if (col0 + 64 < ro.db) tma_store_4d(&maps.out[role], src + 8192, col0 + 64, t0, h, b);
                }
                bulk_commit();
            }
        }
        if (!SUMS) {
            if (warp == SW + VW && lane == 0) bulk_wait();
            if (to == INT_MAX) dla_zero_tail<BF16>(w, ro, b, h, col0, ro.db - col0 < 128 ? ro.db - col0 : 128, chunks * C, seg, tid - 32 * (SW + VW), 32 * OW);
        }
    } else if (warp >= SW) {                                 // v: column `row`, 32 tokens from i0 on
        if (V_REGS < LAUNCH_REGS) regs_dec<V_REGS>();
        const int quad = warp & 3, half = (warp - SW) >> 2, row = quad * 32 + lane, i0 = half * 32;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        for (int c = 0; c < todo; ++c) {
            const int s = c % L::STAGES;
            const bool part = partial(c);
            unsigned char* const tile = ringp + s * L::BYTES;
            unsigned char* const vt = tile + L::V + (row / 64) * 8192 + i0 * 128;
            const float* const add = ctl.add[part] + i0;
            mbar_wait_or_dead(bar(B_FULL + s), (c / L::STAGES) & 1, dead);
            __syncwarp();
            if (part) {                                      // rows past the length: zeros, whatever was there
                for (int p = tid - 32 * SW; p < (C - last_n) * (DA / 8 + 16); p += 32 * VW) {
                    const int rw = last_n + p / (DA / 8 + 16), x = p % (DA / 8 + 16), k = x - 16;
                    *reinterpret_cast<uint4*>(tile + (x < 16 ? L::V + (x / 8) * 8192 : L::RK + (k / 8) * 16384 + 8192) + rw * 128 + (x % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async();
                asm volatile("bar.sync 2, %0;\n" ::"n"(32 * VW) : "memory");
                if (lane == 0) mbar_arrive(bar(B_ZERO));     // once: a walk has one partial chunk
            }
            uint32_t u[3][16];                               // the parts, two tokens in a word
            float2 left = make_float2(0.f, 0.f);             // not 0 where a value is not finite
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const float4 g = *reinterpret_cast<const float4*>(add + 2 * j);
                float2 f[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int i = 2 * (j + e);
                    f[e] = make_float2(load_bf16(vt + sw128_at(i, row % 64)), load_bf16(vt + sw128_at(i + 1, row % 64)));
                    f[e] = __fmul2_rn(e ? make_float2(g.z, g.w) : make_float2(g.x, g.y), f[e]);
                    u[0][j + e] = part2(f[e]);
                    u[1][j + e] = part2(f[e]);
                    u[2][j + e] = pack2(f[e].x, f[e].y);
                    left = __ffma2_rn(f[e], make_float2(0.f, 0.f), left);
                }
            }
            const bool odd = !(left.x + left.y == 0.f);
            int first = reverse ? -1 : C;
            if (__any_sync(0xffffffffu, odd)) {              // g v is not finite and makes its column of D so; v goes
                if (odd) {
#pragma unroll 1
                    for (int j = 0; j < 32; ++j) {
                        unsigned short* const p = reinterpret_cast<unsigned short*>(vt + sw128_at(j, row % 64));
                        if ((*p & 0x7f80u) != 0x7f80u) continue;
                        first = reverse ? max(first, i0 + j) : min(first, i0 + j);
                        *p = 0;
                    }
                }
                fence_async();
            }
            if (!SUMS) ctl.first[c & 3][half][row] = static_cast<short>(first);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_FREE + s));
            if (c > 0) await(bar(B_D + DA / 64 - 1), (c - 1) & 1, dead);
#pragma unroll
            for (int p = 0; p < 3; ++p)
                if (p < parts) tmem_st16(lanes + V_COL + 32 * p + i0 / 2, u[p]);
            announce(bar(B_V), lane);
        }
    } else {                                                 // the state: column `row`, half of da
        regs_inc<STATE_REGS>();
        const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane, col = col0 + row;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        constexpr int RD = DA / 2;                           // rows of da of a warp
        const int x0 = half * RD, da = ro.da, db = ro.db;
        const bool live = col < db;
        const int64_t per = static_cast<int64_t>(ro.width) * db;
        const int64_t at = ro.transposed ? static_cast<int64_t>(col) * ro.width + ro.x0 : static_cast<int64_t>(ro.x0) * db + col, step = ro.transposed ? 1 : db;
        float2 S[RD / 2];
        auto read = [&](const float* p) {
            const float* q = p + at + x0 * step;
#pragma unroll
            for (int x = 0; x < RD / 2; ++x) {
                if (x % 16 == 0) asm volatile("" ::: "memory");      // 32 values in flight, and no more registers
                const bool on = live && x0 + 2 * x < da && p != nullptr;     // da is a multiple of 8
                S[x] = make_float2(on ? __ldcg(q) : 0.f, on ? __ldcg(q + step) : 0.f);
                q += 2 * step;
            }
        };
        auto write = [&](float* p) {
#pragma unroll
            for (int x = 0; x < RD / 2; ++x) {
                const int r = x0 + 2 * x;
                if (live && r < da) {
                    p[at + r * step] = S[x].x;
                    p[at + (r + 1) * step] = S[x].y;
                }
            }
        };
        // Pieces: [0] is the first state, [s + 1] what segment s adds, and for the second launch the state after it.
        float* const pieces = w.seg_state + w.seg_role[role] + chain * w.segs * per;
        if (SUMS) {
            if (seg == 0) {
                read(ro.state_in == nullptr ? nullptr : ro.state_in + chain * per);
                write(pieces);
            }
#pragma unroll
            for (int x = 0; x < RD / 2; ++x) S[x] = make_float2(0.f, 0.f);
        } else {
            if (from == 0) {
                read(w.segs > 1 ? pieces + seg * per : ro.state_in == nullptr ? nullptr : ro.state_in + chain * per);
            } else {                                         // what the chain's first piece left
                if (lane == 0) {
                    unsigned ready = 0;
                    for (int i = w.cut_polls; i > 0 && ready == 0; --i) {
                        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];\n" : "=r"(ready) : "l"(&space->ready[cut]) : "memory");
                        if (ready == 0) __nanosleep(100);
                    }
                    if (ready == 0) *dead = 1;
                }
                __syncwarp();
                const float* p = space->state[cut] + x0 * 128 + row;
#pragma unroll
                for (int x = 0; x < RD / 2; ++x) {
                    if (x % 16 == 0) asm volatile("" ::: "memory");
                    S[x] = make_float2(__ldcg(p + 256 * x), __ldcg(p + 256 * x + 128));
                }
            }
        }
        auto put = [&]() {                                   // S before the next chunk
            if (!SUMS) {
#pragma unroll
                for (int x = 0; x < RD / 2; x += 8) {
                    uint32_t u[8], l[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float2 f = S[x + j];
                        u[j] = part2(f);
                        l[j] = pack2(f.x, f.y);
                    }
                    tmem_st8(lanes + S_COL + x0 / 2 + x, u);
                    tmem_st8(lanes + S_COL + SB + x0 / 2 + x, l);
                }
                announce(bar(B_S), lane);
            }
        };
        if (todo > 0) put();
        for (int c = 0; c < todo; ++c) {
            const float* const lam = ctl.lam[partial(c)];
            const float2 hi = make_float2(lam[0], lam[0]), lo = make_float2(lam[1], lam[1]);
            const int hd = DA > 64 ? half : 0;
            const uint32_t dcol = lanes + D_COL + (DA > 64 ? 0 : x0);
            await(bar(B_D + hd), c & 1, dead);
            float d[2][16];                                  // the next 16 rows are on their way
            tmem_ld16_begin(dcol, d[0]);
#pragma unroll
            for (int x = 0; x < RD / 2; x += 8) {
                float (&dx)[16] = d[x / 8 % 2];
                tmem_ld_wait(dx);
                if (x + 8 < RD / 2) tmem_ld16_begin(dcol + 2 * (x + 8), d[(x / 8 + 1) % 2]);
#pragma unroll
                for (int j = 0; j < 8; ++j) S[x + j] = __ffma2_rn(hi, S[x + j], __ffma2_rn(lo, S[x + j], make_float2(dx[2 * j], dx[2 * j + 1])));
            }
            tc_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_DFREE + hd));
            if (c + 1 < todo) {
                if (!SUMS) await(bar(B_SFREE), c & 1, dead);
                put();
            }
        }
        if (!SUMS && to != INT_MAX) {                        // a first piece
            float* p = space->state[cut] + x0 * 128 + row;
#pragma unroll
            for (int x = 0; x < RD / 2; ++x) {
                p[256 * x] = S[x].x;
                p[256 * x + 128] = S[x].y;
            }
            __threadfence();
            asm volatile("bar.sync 3, %0;\n" ::"n"(32 * SW) : "memory");
            if (tid == 0 && !w.cut_hold) asm volatile("st.release.gpu.global.u32 [%0], 1;\n" ::"l"(&space->ready[cut]) : "memory");
        }
        float* const out = SUMS ? pieces + (seg + 1) * per : ro.state_out != nullptr ? ro.state_out + chain * per : nullptr;
        if (out != nullptr && (SUMS || (seg == w.segs - 1 && to == INT_MAX))) write(out);
    }
    tc_before_sync();
    __syncthreads();
    if (tid == 0 && ctl.dead) flag_error(w.err, ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, T_COLS);
}

template <int DA, bool SUMS>
cudaError_t scan(const ScanMaps& maps, const DlaWalk& w, const ScanCuts& cuts, cudaStream_t stream) {
    constexpr size_t smem = scan_smem<DA>();
    static std::atomic<int> regs{0};
    cudaError_t e = check_kernel_registers(k_dla_scan<DA, SUMS>, LAUNCH_REGS, regs);
    if (e != cudaSuccess) return e;
    static std::atomic<unsigned long long> seen;
    e = allow_smem(k_dla_scan<DA, SUMS>, smem, seen);
    if (e != cudaSuccess) return e;
    int n = 0;
    for (int i = 0; i < w.roles; ++i) n += w.slices[i];
    const unsigned segs = static_cast<unsigned>(SUMS ? w.segs - 1 : w.segs);
    const dim3 grid = cuts.n > 0 ? dim3(static_cast<unsigned>(n) * w.H * w.B + cuts.n) : dim3(n * segs, w.H, w.B);
    k_dla_scan<DA, SUMS><<<grid, ST, smem, stream>>>(maps, w, cuts);
    return cudaGetLastError();
}
template <int DA>
cudaError_t scans(const ScanMaps& maps, const DlaWalk& w, const ScanCuts& cuts, cudaStream_t stream) {
    if (w.segs > 1) {
        cudaError_t e = scan<DA, true>(maps, w, cuts, stream);
        if (e == cudaSuccess) e = launch_dla_prefix(w, C, stream);
        if (e != cudaSuccess) return e;
    }
    return scan<DA, false>(maps, w, cuts, stream);
}

}  // namespace

// A chunk costs the same however few tokens it holds, and however narrow the heads are below 64.  Forward (backward) with 16
// heads of 128, 8 tokens: 21 (93) us against 48 (123) in the fp32 walk at B = 16, 64 (343) against 167 (460) at B = 64; 100
// tokens: 25 (108) against 144 (408) and 87 (386) against 530 (1,554).  Heads of 32, B = 64: 56 (157) against 27 (66) with 8 tokens,
// 50 (142) against 46 (122) with 64, 64 (189) against 74 (201) with 100.
bool dla_scan_pays(int dtype, int T, int dk, int dv) { return dtype == SDM_BF16 && T > 0 && (dk > 64 || dv > 64 || T >= 64); }

namespace {

int64_t scan_ctas(const DlaWalk& w) {
    int64_t ctas = 0;
    for (int i = 0; i < w.roles; ++i) ctas += (w.role[i].db + 127) / 128;
    return ctas * w.B * w.H;
}

}  // namespace

// With fewer CTAs than half of the SMs the tokens are cut, so that every SM has a piece, where that pays: a chunk takes 1.9 us
// in the walk and about 1.1 in the walk for the sums, which with the joining launch costs 10 us more to begin with.  The rule goes by T: a
// piece past the end of a short sequence has nothing to do, and the longest sequence's pieces take as long as if all had its length.
//
// More CTAs than SMs are spread over these where the last round's time that this saves is more than its costs: about 6 us for the
// cut chains' extra starts, and 1 us for every CTA's number.  Forward (backward), 10 x 16 heads of 128: 256 -> 154 us (532 -> 458)
// with 64 chunks, 60 (30) of which are saved, 136 -> 93 (300 -> 274) with 32, 76 -> 60 (180 -> 174) with 16, where it is 15 (13); 133 -> 138
// backward with 10, where it is 8; 80 x 16 heads, 16 chunks, backward, 11 saved in 26 rounds: 1,158 -> 1,182.
void dla_scan_plan(DlaWalk& w) {
    const int64_t ctas = scan_ctas(w), chunks = (w.T + C - 1) / C;
    int64_t segs = SMS / ctas;
    if (segs > chunks / 2) segs = chunks / 2;
    if (segs < 2 || chunks * (2 * segs - 3) <= 10 * segs) segs = 1;
    w.seg_chunks = static_cast<int>((chunks + segs - 1) / segs);
    w.segs = static_cast<int>((chunks + w.seg_chunks - 1) / w.seg_chunks);
    const int64_t span = (ctas * chunks + SMS - 1) / SMS, rounds = (ctas + SMS - 1) / SMS;
    w.span = ctas > SMS && rounds * chunks - span >= SPREAD_SAVES + rounds / 2 ? static_cast<int>(span) : 0;
    w.cut_polls = 4 * 1000 * 1000 + 32 * static_cast<int>(chunks);      // a first piece takes 2.1 us a chunk
}
size_t dla_scan_cut_bytes() { return sizeof(CutSpace); }

namespace {

ScanCuts scan_cuts(const DlaWalk& w) {
    ScanCuts c{};
    if (w.span == 0) return c;
    const int64_t total = scan_ctas(w) * ((w.T + C - 1) / C), chunks = (w.T + C - 1) / C;
    for (int64_t p = w.span; p < total && c.n < SMS; p += w.span) {
        const int rest = static_cast<int>(p % chunks);       // behind the SM's own chains; the piece before it is the next SM's first
        if (rest < CUT_LEAST || chunks - rest < CUT_LEAST) continue;
        c.chain[c.n] = static_cast<int>(p / chunks);
        c.at[c.n] = static_cast<int>(chunks - rest);
        c.order[c.n] = static_cast<short>(c.n);
        ++c.n;
    }
    std::sort(c.order, c.order + c.n, [&](short a, short b) { return c.at[a] != c.at[b] ? c.at[a] < c.at[b] : a < b; });
    return c;
}

}  // namespace

int dla_scan_cuts(const DlaWalk& w) { return scan_cuts(w).n; }

cudaError_t launch_dla_scan(DlaWalk& w, cudaStream_t stream) {
    ScanMaps m;
    int da = 0;
    for (int i = 0; i < w.roles; ++i) {
        const DlaRole& r = w.role[i];
        da = r.da > da ? r.da : da;
        w.slices[i] = (r.db + 127) / 128;
        if (!token_map(&m.r[i], r.r, w.token_major, w.B, r.hr, w.T, r.width) || !token_map(&m.k[i], r.k, w.token_major, w.B, r.hk, w.T, r.width) ||
            !token_map(&m.v[i], r.v, w.token_major, w.B, r.hv, w.T, r.db) ||
            (!r.partial && !token_map(&m.out[i], r.out, w.token_major, w.B, w.H, w.T, r.db)))
            return cudaErrorInvalidValue;
    }
    const ScanCuts cuts = scan_cuts(w);
    if (cuts.n == 0) {
        w.span = 0;
    } else {
        const cudaError_t e = cudaMemsetAsync(w.seg_state, 0, offsetof(CutSpace, state), stream);
        if (e != cudaSuccess) return e;
    }
    return da <= 64 ? scans<64>(m, w, cuts, stream) : scans<128>(m, w, cuts, stream);
}

}  // namespace sdm
