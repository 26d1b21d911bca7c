// Linear attention with a decay per head on the tensor cores: bf16, widths of the contraction up to 128, chunks of 64 tokens.
//
// A CTA walks one state, 128 columns of it (db), over its chunks; every product has 128 rows, TMEM lanes = columns of the state:
//   1  P[i, j]  = r_i.k_j                       A = [r; k] in shared memory (the k half is not used), B = k
//   2  I[c, i]  = sum_x S[x, c] r_i[x]          A = S transposed, two bf16 parts in TMEM
//   3  O[c, i]  = sum_j v_j[c] W_ij P_ij        A = v transposed in TMEM, B = the weighted P as two bf16 parts in shared memory
//   4  D[c, x]  = sum_j g_j v_j[c] k_j[x]       A = g v transposed, three bf16 parts in TMEM, B = k
// and out_i = w_i I + O, S <- lam^n S + D, in float32 and with lam^n in two parts.  W, w and g hold the powers of the decay
// (dla_internal.h).  r and k are used as TMA leaves them; v goes through registers, which transposes it, scales it and keeps
// what lies past the length out of the products.
//
// bf16 parts: g v has 8 + 24 significant bits, three parts keep 24 of them, so that the state is as good as a float32
// sum; S and the weighted P only reach outputs that are rounded to 2^-9, and two parts keep 16 bits.
//
// Only D goes from one chunk to the next, and it does not depend on S: six groups of warps work on different stages of
// neighbouring chunks, each handing over through mbarriers.
//
// A value of v that is not finite must stay out of the outputs before its token, which share its products: v is zero in
// them from that token on, its column's outputs from there are NaN, and so is the column of the state.
#include "dla_internal.h"
#include "gdn_tc.cuh"
#include "sdm_common.cuh"

namespace sdm {

namespace {

using namespace gdn;

constexpr int SW = 8, VW = 4, OW = 4, PW = 4;  // warps: state, v, outputs, and (the last four) P, P, products, copies
constexpr int ST = 32 * (SW + VW + OW + PW);
constexpr int LAUNCH_REGS = 96, STATE_REGS = 120, REST_REGS = 80;
static_assert(SW * STATE_REGS + (VW + OW + PW) * REST_REGS <= (SW + VW + OW + PW) * LAUNCH_REGS, "register split");

// TMEM columns.  O lies where P was.
constexpr uint32_t S_COL = 0, D_COL = 128, V_COL = 256, P_COL = 384, I_COL = 448, T_COLS = 512;
constexpr int WP = 68;                         // floats of a row of W, so that rows start four banks apart

template <int DA>
struct ScanTile {
    static constexpr uint32_t RK = 0, V = DA / 64 * 16384, BYTES = V + 16384;        // [r; k] per 64 of da; v per 64 columns
    static constexpr int STAGES = DA == 128 ? 3 : 4;
    static constexpr uint32_t PS = BYTES * STAGES, OUT = PS + 2 * MAT, CTL = OUT + 2 * 16384;
};
enum { B_FULL = 0, B_FREE = 4, B_P = 8, B_PS, B_D, B_D2, B_O, B_VFREE, B_V, B_OFREE, B_S, B_COUNT };
struct ScanCtl {
    float W[C * WP];
    float add[2][C], inter[2][C];              // weights of a whole chunk and of the partial one
    float pw[C + 1];
    float lam[2][2];                           // lam^n of both in two parts
    short first[2][128];                       // of a column: the chunk's first value (in the walk's order) that is not finite
    unsigned long long bar[B_COUNT];
    uint32_t tmem;
    int dead;
};
template <int DA>
constexpr size_t scan_smem() { return 1024 + ScanTile<DA>::CTL + sizeof(ScanCtl); }
static_assert(scan_smem<128>() <= 227 * 1024 && scan_smem<64>() <= 227 * 1024, "shared memory");

struct ScanMaps {
    CUtensorMap r[3], k[3], v[3], out[3];
};

// The upper halves of two floats as a pair of bf16, and what they leave.
__device__ __forceinline__ uint32_t cut2(float2& v) {
    const uint32_t x = __float_as_uint(v.x), y = __float_as_uint(v.y);
    const float2 hi = make_float2(__uint_as_float(x & 0xffff0000u), __uint_as_float(y & 0xffff0000u));
    v = __ffma2_rn(hi, make_float2(-1.f, -1.f), v);
    return __byte_perm(x, y, 0x7632);
}

template <int DA, bool SUMS>
__global__ void __launch_bounds__(ST, 1) k_dla_scan(const __grid_constant__ ScanMaps maps, const __grid_constant__ DlaWalk w, const int3 slices) {
    using L = ScanTile<DA>;
    extern __shared__ unsigned char raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t ring = (base + 1023u) & ~1023u;
    unsigned char* const ringp = raw + (ring - base);
    ScanCtl& ctl = *reinterpret_cast<ScanCtl*>(ringp + L::CTL);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int nseg = SUMS ? w.segs - 1 : w.segs, seg = blockIdx.x % nseg;
    int slice = blockIdx.x / nseg, role = 0;
    if (slice >= slices.x) {
        slice -= slices.x;
        role = 1;
        if (slice >= slices.y) {
            slice -= slices.y;
            role = 2;
        }
    }
    const DlaRole& ro = w.role[role];
    const int b = blockIdx.z, h = blockIdx.y, col0 = slice * 128;
    const int len = dla_length(w, b), chunks = (len + C - 1) / C;
    const bool reverse = ro.reverse != 0;
    const int c0 = min(seg * w.seg_chunks, chunks), c1 = seg == w.segs - 1 ? chunks : min(c0 + w.seg_chunks, chunks);
    const int todo = c1 - c0, last_n = len - (chunks - 1) * C;       // tokens of the sequence's last chunk
    auto chunk_at = [&](int c) { return reverse ? chunks - 1 - (c0 + c) : c0 + c; };
    auto partial = [&](int c) { return chunk_at(c) == chunks - 1 && last_n < C; };
    const int64_t chain = static_cast<int64_t>(b) * w.H + h;
    const float ld = __ldg(w.log_decay + h);
    const uint32_t bars = smem_u32(&ctl.bar[0]);
    auto bar = [&](int i) { return bars + 8 * i; };
    if (tid == 0) {
        ctl.dead = 0;
        for (int i = 0; i < B_COUNT; ++i)
            mbar_init(bar(i), i >= B_FREE && i < B_P ? VW + 1 : i == B_PS ? 2 : i == B_V ? VW : i == B_OFREE ? OW : i == B_S ? SW : 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
    }
    if (warp == 0) tmem_alloc(smem_u32(&ctl.tmem), T_COLS);
    if (tid <= C) ctl.pw[tid] = dla_pow(ld, tid);
    if (tid >= 96 && tid < 98) {
        const int n = tid == 96 ? C : last_n;
        const double f = n == 0 ? 1.0 : exp(static_cast<double>(n) * static_cast<double>(ld));
        const float hi = static_cast<float>(f), lo = static_cast<float>(f - static_cast<double>(hi));
        ctl.lam[tid - 96][0] = hi;
        ctl.lam[tid - 96][1] = gdn_finite(hi) ? lo : 0.f;
    }
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
            for (int c = 0; !SUMS && c < todo; ++c) {
                await(bar(B_P), c & 1, dead);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float p[32];
                    tmem_ld32(lanes + P_COL + 32 * e, p);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t u[4], l[4];
                        const float4 wa = *reinterpret_cast<const float4*>(wt + 32 * e + 8 * q), wb = *reinterpret_cast<const float4*>(wt + 32 * e + 8 * q + 4);
                        const float ww[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            // zero by choice: a token past this one may not be finite
                            float2 f = make_float2(ww[2 * s] != 0.f ? ww[2 * s] * p[8 * q + 2 * s] : 0.f,
                                                   ww[2 * s + 1] != 0.f ? ww[2 * s + 1] * p[8 * q + 2 * s + 1] : 0.f);
                            u[s] = cut2(f);
                            l[s] = pack2(f.x, f.y);
                        }
                        unsigned char* const at = ps + box_at(i, 4 * e + q);
                        *reinterpret_cast<uint4*>(at) = make_uint4(u[0], u[1], u[2], u[3]);
                        *reinterpret_cast<uint4*>(at + MAT) = make_uint4(l[0], l[1], l[2], l[3]);
                    }
                }
                tc_before_sync();
                hand_over(bar(B_PS), lane);
            }
        } else if (me == 2) {                                // products
            const uint32_t id64 = mma_idesc(64);
            for (int c = 0; c < todo; ++c) {
                const int s = c % L::STAGES;
                const uint32_t t = ring + s * L::BYTES, ph = c & 1;
                const uint64_t dr = sw128_desc(t + L::RK), dk = sw128_desc(t + L::RK + 8192), dkt = sw128_mn_desc(t + L::RK + 8192, 16384),
                               dp = sw128_desc(ring + L::PS);
                await(bar(B_FULL + s), (c / L::STAGES) & 1, dead);
                if (!SUMS) {
                    if (partial(c)) await(bar(B_V), ph, dead);       // k's rows past the length are zero by then
                    if (c > 0) await(bar(B_OFREE), (c - 1) & 1, dead);
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < DA / 16; ++kk)
                            mma_bf16(tmem + P_COL, dr + (kk / 4) * 1024 + (kk % 4) * 2, dk + (kk / 4) * 1024 + (kk % 4) * 2, id64, kk != 0);
                        mma_commit(bar(B_P));
                    }
                    __syncwarp();
                }
                await(bar(B_S), ph, dead);
                if (!SUMS && elect_one()) {                  // lower parts first, here and below: their sums are small
#pragma unroll 1
                    for (int p = 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < DA / 16; ++kk)
                            mma_bf16_ta(tmem + I_COL, tmem + S_COL + p * SB + kk * 8, dr + (kk / 4) * 1024 + (kk % 4) * 2, id64, p != 1 || kk != 0);
                }
                __syncwarp();
                await(bar(B_V), ph, dead);
                if (elect_one()) {
#pragma unroll 1
                    for (int x = 0; x < DA / 64; ++x) {
#pragma unroll 1
                        for (int p = 2; p >= 0; --p)
#pragma unroll
                            for (int kk = 0; kk < C / 16; ++kk)
                                mma_bf16_ta(tmem + D_COL + x * 64, tmem + V_COL + 32 + p * 32 + kk * 8, dkt + x * 1024 + kk * 128, id64 | MN_B, p != 2 || kk != 0);
                        mma_commit(bar(B_D + x));
                    }
                    if (DA == 64) mma_commit(bar(B_D2));
                    if (SUMS) {
                        mma_commit(bar(B_VFREE));
                        mma_commit(bar(B_FREE + s));
                    }
                }
                __syncwarp();
                if (SUMS) continue;
                await(bar(B_PS), ph, dead);
                if (elect_one()) {
#pragma unroll 1
                    for (int p = 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + P_COL, tmem + V_COL + kk * 8, dp + p * (MAT / 16) + kk * 2, id64, p != 1 || kk != 0);
                    mma_commit(bar(B_O));
                    mma_commit(bar(B_VFREE));
                    mma_commit(bar(B_FREE + s));
                }
                __syncwarp();
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
                    tma_load_4d(t + L::RK + x * 16384 + 8192, &maps.k[role], 64 * x, at, hk, b, fb);
                    if (!SUMS) tma_load_4d(t + L::RK + x * 16384, &maps.r[role], 64 * x, at, hr, b, fb);
                }
                tma_load_4d(t + L::V, &maps.v[role], col0, at, hv, b, fb);
                tma_load_4d(t + L::V + 8192, &maps.v[role], col0 + 64, at, hv, b, fb);
            }
            if (*dead)                                       // the copies in flight land before the CTA ends
                for (int j = loaded > L::STAGES ? loaded - L::STAGES : 0; j < loaded; ++j)
                    mbar_wait(bar(B_FULL + j % L::STAGES), (j / L::STAGES) & 1);
        }
    } else if (warp >= SW + VW) {                            // outputs: column `row`, all tokens
        regs_dec<REST_REGS>();
        const int quad = warp & 3, row = quad * 32 + lane, col = col0 + row;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const bool share = ro.partial != 0;
        float* const shares = static_cast<float*>(ro.out) + chain * w.T * ro.db + col;
        for (int c = 0; !SUMS && c < todo; ++c) {
            const bool part = partial(c);
            const int n = part ? last_n : C, t0 = chunk_at(c) * C;
            unsigned char* const box = ringp + L::OUT + (c & 1) * 16384;
            unsigned char* const yt = box + (row / 64) * 8192;
            const float* const wi = ctl.inter[part];
            if (!share) {                                    // the copy before the last has left this box
                if (warp == SW + VW && lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;\n" ::: "memory");
                asm volatile("bar.sync 1, %0;\n" ::"n"(32 * OW) : "memory");
            }
            await(bar(B_O), c & 1, dead);
            const int first = ctl.first[c & 1][row];
            const bool odd = __any_sync(0xffffffffu, first != (reverse ? -1 : C));
#pragma unroll
            for (int e = 0; e < 4; ++e) {                    // 16 tokens at a time
                float y[16], o[16];
                tmem_ld16(lanes + I_COL + 16 * e, y);
                tmem_ld16(lanes + P_COL + 16 * e, o);
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
                        const int i = 16 * e + j;
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
            if (seg == w.segs - 1 && col < ro.db) {          // chunks past the length
                __nv_bfloat16* y = static_cast<__nv_bfloat16*>(ro.out) + gdn_base(w.token_major, b, h, w.H, w.T, ro.db) + col;
                const int64_t ys = gdn_stride(w.token_major, w.H, ro.db);
                for (int64_t t = static_cast<int64_t>(chunks) * C; t < w.T; ++t) {
                    if (share) shares[t * ro.db] = 0.f;
                    else y[t * ys] = __float2bfloat16_rn(0.f);
                }
            }
        }
    } else if (warp >= SW) {                                 // v: column `row`, all tokens
        regs_dec<REST_REGS>();
        const int quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const bool live = col0 + row < ro.db;
        for (int c = 0; c < todo; ++c) {
            const int s = c % L::STAGES;
            const bool part = partial(c);
            const int n = part ? last_n : C;
            unsigned char* const tile = ringp + s * L::BYTES;
            const unsigned char* const vt = tile + L::V + (row / 64) * 8192;
            const float* const add = ctl.add[part];
            mbar_wait_or_dead(bar(B_FULL + s), (c / L::STAGES) & 1, dead);
            __syncwarp();
            uint32_t v[C / 2];                               // two tokens in a word
#pragma unroll
            for (int j = 0; j < C / 2; ++j)
                v[j] = *reinterpret_cast<const unsigned short*>(vt + sw128_at(2 * j, row % 64)) |
                       (static_cast<uint32_t>(*reinterpret_cast<const unsigned short*>(vt + sw128_at(2 * j + 1, row % 64))) << 16);
            if (part) {                                      // v and the rows of k past the length: zeros, whatever was there
#pragma unroll
                for (int j = 0; j < C / 2; ++j) v[j] &= 2 * j + 1 < n ? 0xffffffffu : 2 * j < n ? 0x0000ffffu : 0u;
                for (int p = tid - 32 * SW; p < (C - n) * DA / 8; p += 32 * VW) {
                    const int rw = n + p / (DA / 8), x = p % (DA / 8);
                    *reinterpret_cast<uint4*>(tile + L::RK + (x / 8) * 16384 + 8192 + rw * 128 + (x % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_FREE + s));
            uint32_t top = 0;                                // the largest exponent
#pragma unroll
            for (int j = 0; j < C / 2; ++j) top = __vmaxu2(top, v[j] & 0x7fff7fffu);
            const bool mine = live && ((top & 0xffffu) >= 0x7f80u || (top >> 16) >= 0x7f80u);
            const bool odd = __any_sync(0xffffffffu, mine);
            int first = reverse ? -1 : C;
            if (odd) {
                if (mine) {
#pragma unroll
                    for (int j = 0; j < C; ++j)
                        if (((v[j / 2] >> (j % 2 * 16)) & 0x7f80u) == 0x7f80u) first = reverse ? max(first, j) : min(first, j);
                }
#pragma unroll
                for (int j = 0; j < C; ++j)
                    if (reverse ? j <= first : j >= first) v[j / 2] &= j % 2 ? 0x0000ffffu : 0xffff0000u;
            }
            if (c > 0) await(bar(B_VFREE), (c - 1) & 1, dead);
            if (!SUMS) {
                ctl.first[c & 1][row] = static_cast<short>(first);
                uint32_t u[16];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) u[j] = v[16 * e + j];
                    tmem_st16(lanes + V_COL + 16 * e, u);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {                    // 16 tokens at a time
                float2 f[8];
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const float4 g = *reinterpret_cast<const float4*>(add + 16 * e + 2 * j);
                    const uint32_t a = v[8 * e + j], d = v[8 * e + j + 1];
                    f[j] = __fmul2_rn(make_float2(g.x, g.y), make_float2(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u)));
                    f[j + 1] = __fmul2_rn(make_float2(g.z, g.w), make_float2(__uint_as_float(d << 16), __uint_as_float(d & 0xffff0000u)));
                }
                if (odd) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int i = 16 * e + 2 * j;
                        if (reverse ? i <= first : i >= first) f[j].x = gdn_nan();
                        if (reverse ? i + 1 <= first : i + 1 >= first) f[j].y = gdn_nan();
                    }
                }
                uint32_t u[8];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) u[j] = cut2(f[j]);
                    tmem_st8(lanes + V_COL + 32 + 32 * p + 8 * e, u);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = pack2(f[j].x, f[j].y);
                tmem_st8(lanes + V_COL + 96 + 8 * e, u);
            }
            announce(bar(B_V), lane);
        }
    } else {                                                 // the state: column `row`, half of da
        regs_inc<STATE_REGS>();
        const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane, col = col0 + row;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        constexpr int RD = DA / 2;                           // rows of da of a warp
        const int x0 = half * RD, da = ro.da, db = ro.db;
        const bool live = col < db;
        const int64_t per = static_cast<int64_t>(da) * db;
        const int64_t at = ro.transposed ? static_cast<int64_t>(col) * da : col, step = ro.transposed ? 1 : db;
        float2 S[RD / 2];
        // `keep` times S plus the state at p
        auto read = [&](const float* p, float keep, bool start) {
#pragma unroll
            for (int x = 0; x < RD / 2; ++x) {
                const int r = x0 + 2 * x;                    // da is a multiple of 8
                const bool on = live && r < da && p != nullptr;
                const float a = on ? __ldcg(p + at + r * step) : 0.f, d = on ? __ldcg(p + at + (r + 1) * step) : 0.f;
                S[x] = start ? make_float2(a, d) : make_float2(fmaf(keep, S[x].x, a), fmaf(keep, S[x].y, d));
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
        // Pieces: [0] is the first state, [s + 1] what segment s adds.
        float* const pieces = w.seg_state + w.seg_role[role] + chain * w.segs * per;
        if (SUMS) {
            if (seg == 0) {
                read(ro.state_in == nullptr ? nullptr : ro.state_in + chain * per, 0.f, true);
                write(pieces);
            }
#pragma unroll
            for (int x = 0; x < RD / 2; ++x) S[x] = make_float2(0.f, 0.f);
        } else if (w.segs == 1) {
            read(ro.state_in == nullptr ? nullptr : ro.state_in + chain * per, 0.f, true);
        } else {
            read(pieces, 0.f, true);
            const float full = dla_pow(ld, w.seg_chunks * C);
            for (int s = 0; s < seg; ++s) {
                const int s0 = min(s * w.seg_chunks, chunks), s1 = min(s0 + w.seg_chunks, chunks);
                if (s0 == s1) break;
                int n = (s1 - s0) * C;                       // the walk's partial chunk is the sequence's last
                if (reverse ? s0 == 0 : s1 == chunks) n -= C - last_n;
                read(pieces + (s + 1) * per, n == w.seg_chunks * C ? full : dla_pow(ld, n), false);
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
                        u[j] = cut2(f);
                        l[j] = pack2(f.x, f.y);
                    }
                    tmem_st8(lanes + S_COL + x0 / 2 + x, u);
                    tmem_st8(lanes + S_COL + SB + x0 / 2 + x, l);
                }
            }
            announce(bar(B_S), lane);
        };
        if (todo > 0) put();
        for (int c = 0; c < todo; ++c) {
            const float* const lam = ctl.lam[partial(c)];
            const float2 hi = make_float2(lam[0], lam[0]), lo = make_float2(lam[1], lam[1]);
            await(bar(B_D + half), c & 1, dead);
#pragma unroll
            for (int x = 0; x < RD / 2; x += 8) {
                float d[16];
                tmem_ld16(lanes + D_COL + x0 + 2 * x, d);
#pragma unroll
                for (int j = 0; j < 8; ++j) S[x + j] = __ffma2_rn(hi, S[x + j], __ffma2_rn(lo, S[x + j], make_float2(d[2 * j], d[2 * j + 1])));
            }
            if (c + 1 < todo) {
                tc_before_sync();
                put();
            }
        }
        float* const out = SUMS ? pieces + (seg + 1) * per : ro.state_out != nullptr ? ro.state_out + chain * per : nullptr;
        if (out != nullptr && (SUMS || seg == w.segs - 1)) write(out);
    }
    tc_before_sync();
    __syncthreads();
    if (tid == 0 && ctl.dead) flag_error(w.err, ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, T_COLS);
}

template <int DA, bool SUMS>
cudaError_t scan(const ScanMaps& maps, const DlaWalk& w, cudaStream_t stream) {
    constexpr size_t smem = scan_smem<DA>();
    static std::atomic<int> regs{0};
    cudaError_t e = check_kernel_registers(k_dla_scan<DA, SUMS>, LAUNCH_REGS, regs);
    if (e != cudaSuccess) return e;
    static std::atomic<unsigned long long> seen;
    e = allow_smem(k_dla_scan<DA, SUMS>, smem, seen);
    if (e != cudaSuccess) return e;
    int n[3] = {0, 0, 0};
    for (int i = 0; i < w.roles; ++i) n[i] = (w.role[i].db + 127) / 128;
    const unsigned segs = static_cast<unsigned>(SUMS ? w.segs - 1 : w.segs);
    k_dla_scan<DA, SUMS><<<dim3((n[0] + n[1] + n[2]) * segs, w.H, w.B), ST, smem, stream>>>(maps, w, make_int3(n[0], n[1], n[2]));
    return cudaGetLastError();
}
template <int DA>
cudaError_t scans(const ScanMaps& maps, const DlaWalk& w, cudaStream_t stream) {
    if (w.segs > 1) {
        cudaError_t e = scan<DA, true>(maps, w, stream);
        if (e != cudaSuccess) return e;
    }
    return scan<DA, false>(maps, w, stream);
}

int widest(const DlaWalk& w) {
    int da = 0;
    for (int i = 0; i < w.roles; ++i) da = w.role[i].da > da ? w.role[i].da : da;
    return da;
}

}  // namespace

bool dla_scan_supported(int dtype, const DlaWalk& w) { return dtype == SDM_BF16 && widest(w) <= 128 && w.T >= 32; }

void dla_scan_plan(DlaWalk& w) {
    w.segs = 1;
    w.seg_chunks = (w.T + C - 1) / C;
}

cudaError_t launch_dla_scan(const DlaWalk& w, cudaStream_t stream) {
    ScanMaps m;
    for (int i = 0; i < w.roles; ++i) {
        const DlaRole& r = w.role[i];
        if (!token_map(&m.r[i], r.r, w.token_major, w.B, r.hr, w.T, r.da) || !token_map(&m.k[i], r.k, w.token_major, w.B, r.hk, w.T, r.da) ||
            !token_map(&m.v[i], r.v, w.token_major, w.B, r.hv, w.T, r.db) ||
            (!r.partial && !token_map(&m.out[i], r.out, w.token_major, w.B, w.H, w.T, r.db)))
            return cudaErrorInvalidValue;
    }
    return widest(w) <= 64 ? scans<64>(m, w, stream) : scans<128>(m, w, stream);
}

}  // namespace sdm
