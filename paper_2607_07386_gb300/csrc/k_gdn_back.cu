// Gated delta rule in chunks of 64 tokens, the walk of the backward pass (bf16 storage, d_k <= 128): the
// gradient D of the state, from the last chunk to the first.  With B, N, P, g and h of a chunk as in the
// forward (N = -(I + B beta)^-1 B), D the gradient of the state after it and dy scaled:
//   x = h K D + P^T dy                       the gradient of w = beta e, but for what later e take from it
//   d = (I + beta B)^-T x = x + N^T (beta x)
//   dv = beta d,   D' = g_63 D + Q^T (g dy) - K^T (beta g d)
// The layout is the forward walk's: a CTA owns 128 columns of one state, a TMEM lane is a column, every
// product is D^T-like, its A operand written to TMEM from registers.  Per chunk:
//   1  dy^T P, D^T K^T, then (g dy)^T Q              (MMA; the first needs nothing of the chain, the last runs
//                                                    under step 2)
//   2  x = h .. + ..                                 (registers, bf16 parts to TMEM)
//   3  (beta x)^T N                                  (MMA)
//   4  d = x + ..,  beta g d                         (registers, bf16 parts to TMEM)
//   5  .. += (-beta g d)^T K                         (MMA; dv, d and the next chunk's dy are put away meanwhile)
//   6  D = g_63 D + ..                               (registers, bf16 parts to TMEM)
// D before every step 6 (as bf16), d (as two bf16 parts) and the products <D^T k_j, e_j> with the forward's e are stored for the
// gradients of q, k and the gates.
// Operands are split as in the forward, into three bf16 parts, and so is P, which D depends on (with two, 1e-5 of D at keys
// of a cosine of 0.98).
// The chain of the six stages bounds it: 374 us at B = 8, H = 16, T = 4096, 128 x 128, 10,700 cycles a chunk.  It was 280 with
// two parts of D, N, P and beta x, 324 with three; the products with e, whose lane sums give the gradients' kernel back
// 40, are the rest.
#include "gdn_tc.cuh"

namespace sdm {

namespace {

using namespace tc;
using namespace gdn;

constexpr int SW = 8;                          // compute warps: two share a lane quarter
constexpr int ST = 32 * (SW + 4);
constexpr int LAUNCH_REGS = 168, BACK_REGS = 232, IDLE_REGS = 40;   // a thread's registers, at first and after the split
static_assert(BACK_REGS >= LAUNCH_REGS && IDLE_REGS <= LAUNCH_REGS && SW * BACK_REGS + 4 * IDLE_REGS <= (SW + 4) * LAUNCH_REGS, "register split");
constexpr int NP = 3;                          // bf16 parts of D, of beta x and of what is added to D (see the forward walk)
// TMEM columns: X: D^T K^T, then step 3; Z: dy^T P, then beta x; A: the update, and before that, with d_k > 64, the third
// part of D, of every 64 rows in the first 32 of their own columns, which the warp that writes it has read; S: D, then
// beta g d and the third part of beta x; dy; g dy.
constexpr uint32_t X_COL = 0, Z_COL = 64, A_COL = 128, S_COL = 256, Z3_COL = S_COL + 32 * NP, Y_COL = 384, GY_COL = 416, T_COLS = 512;
// Where 16 rows of d_k from x on of part p of D lie.
template <int DK>
__device__ __forceinline__ constexpr uint32_t d_at(int p, int x) {
    return DK == 128 && p == 2 ? A_COL + x / 64 * 64 + x % 64 / 2 : S_COL + p * (DK / 2) + x / 2;
}

template <int DK>
struct BackTile {
    static constexpr uint32_t KQ = 0, Y = 128 * 2 * DK, BYTES = Y + C * 256, LOAD = BYTES + GATES;
    static constexpr int STAGES = 2;
    // N and P in their parts; e, per part; a box of 128 columns on its way to memory (D per 64 of d_k, then d per part);
    // the stages' gate products
    static constexpr uint32_t N = BYTES * STAGES, P = N + GDN_N_PARTS * MAT, E = N + GDN_BACK_MATS * MAT, KS = E + 32768, G = KS + 32768,
                              CTL = G + STAGES * GATES;
};
// Barriers.  Completed by copies: a stage's tile, P, N, e; by MMAs: U, beta x N, the update; by the copying thread: D (all)
// has left the box; by warps: the rest.
enum { B_FULL = 0, B_P = 2, B_N, B_E, B_U, B_XN, B_UP, B_DFREE, B_FREE, B_S, B_DY, B_X, B_H, B_KS, B_OUT, B_COUNT };
struct BackCtl {
    unsigned long long bar[B_COUNT];
    uint32_t tmem;
    int dead;
};
template <int DK>
constexpr size_t back_smem() { return 1024 + BackTile<DK>::CTL + sizeof(BackCtl); }

// Both warps of a lane quarter.
__device__ __forceinline__ void bar_pair(int quad) {
    tc_before_sync();
    asm volatile("bar.sync %0, 64;\n" ::"r"(1 + quad) : "memory");
    tc_after_sync();
}

template <int DK>
__global__ void __launch_bounds__(ST, 1) k_gdn_back(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tq,
                                                    const __grid_constant__ CUtensorMap ty, const __grid_constant__ CUtensorMap tdv,
                                                    const __grid_constant__ CUtensorMap tm, const __grid_constant__ CUtensorMap tD, const __grid_constant__ CUtensorMap td,
                                                    const __grid_constant__ CUtensorMap te,
                                                    const GdnBack r, const GdnFactors f, int nc) {
    using L = BackTile<DK>;
    extern __shared__ unsigned char raw[];
    const GdnArgs& a = r.a;
    const uint32_t base = smem_u32(raw);
    const uint32_t ring = (base + 1023u) & ~1023u;
    unsigned char* const ringp = raw + (ring - base);
    BackCtl& ctl = *reinterpret_cast<BackCtl*>(ringp + L::CTL);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b = blockIdx.z, h = blockIdx.y, col0 = blockIdx.x * 128, hk = h / (a.H / a.Hk);
    const int len = gdn_length(a, b);
    const int64_t chain = static_cast<int64_t>(b) * a.H + h;
    const int chunks = (len + C - 1) / C;
    const uint32_t bars = smem_u32(&ctl.bar[0]);
    auto bar = [&](int i) { return bars + 8 * i; };
    if (tid == 0) {
        ctl.dead = 0;
        for (int i = 0; i < B_COUNT; ++i) mbar_init(bar(i), i < B_S ? 1 : SW);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
    }
    if (warp == 0) tmem_alloc(smem_u32(&ctl.tmem), T_COLS);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = ctl.tmem;
    volatile int* dead = &ctl.dead;

    if (warp >= SW) {
        regs_dec<IDLE_REGS>();
        if (warp == SW) {                                    // MMAs
            const uint32_t id64 = mma_idesc(64), idm = id64 | MN_B, idk = mma_idesc(DK) | MN_B;
            for (int it = 0; it < chunks; ++it) {
                const uint32_t t = ring + (it % L::STAGES) * L::BYTES, ph = it & 1;
                const uint64_t dk = sw128_desc(t + L::KQ), dn = sw128_mn_desc(ring + L::N, 8192), dp = sw128_mn_desc(ring + L::P, 8192),
                               dkt = sw128_mn_desc(t + L::KQ, 16384), dqt = sw128_mn_desc(t + L::KQ + 8192, 16384);
                await(bar(B_FULL + it % L::STAGES), (it / L::STAGES) & 1, dead);
                await(bar(B_P), ph, dead);
                await(bar(B_DY), ph, dead);
                if (elect_one()) {                           // step 1
#pragma unroll 1
                    for (int p = GDN_BACK_MATS - GDN_N_PARTS - 1, first = 0; p >= 0; --p, first = 1)
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + Z_COL, tmem + Y_COL + kk * 8, dp + p * (MAT / 16) + kk * 128, idm, first != 0 || kk != 0);
                }
                __syncwarp();
                await(bar(B_S), ph, dead);
                if (elect_one()) {
#pragma unroll                                               // lower parts first, here and below: their sums are small
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < DK / 16; ++kk)
                            mma_bf16_ta(tmem + X_COL, tmem + d_at<DK>(p, 16 * kk), dk + (kk / 4) * 1024 + (kk % 4) * 2, id64, p != NP - 1 || kk != 0);
                    mma_commit(bar(B_U));
                }
                __syncwarp();
                if (DK == 128) await(bar(B_U), ph, dead);    // D's third part is read
                if (elect_one()) {
#pragma unroll 1
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + A_COL, tmem + GY_COL + p * 32 + kk * 8, dqt + kk * 128, idk, p != NP - 1 || kk != 0);
                }
                __syncwarp();
                await(bar(B_N), ph, dead);
                await(bar(B_X), ph, dead);
                if (elect_one()) {                           // step 3: part xa of beta x with part nb of N
#pragma unroll 1
                    for (int m = 5; m >= 0; --m) {
                        const int xa = m < 5 ? m / 2 : 0, nb = m < 5 ? m % 2 : 2;    // (0, 2), (2, 0), (1, 1), (1, 0), (0, 1), (0, 0)
                        const uint32_t from = xa == 2 ? Z3_COL : Z_COL + xa * 32;
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + X_COL, tmem + from + kk * 8, dn + nb * (MAT / 16) + kk * 128, idm, m != 5 || kk != 0);
                    }
                    mma_commit(bar(B_XN));
                }
                __syncwarp();
                await(bar(B_H), ph, dead);
                if (elect_one()) {                           // step 5
#pragma unroll 1
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int kk = 0; kk < C / 16; ++kk)
                            mma_bf16_ta(tmem + A_COL, tmem + S_COL + p * 32 + kk * 8, dkt + kk * 128, idk, 1);
                    mma_commit(bar(B_UP));
                }
                __syncwarp();
            }
        } else if (warp == SW + 1 && lane == 0) {            // copies
            auto load = [&](int it) {
                const int c = chunks - 1 - it;
                const uint32_t t = ring + (it % L::STAGES) * L::BYTES, fb = bar(B_FULL + it % L::STAGES);
                const int64_t cid = chain * nc + c;
                mbar_expect_tx(fb, L::LOAD);
#pragma unroll
                for (int x = 0; x < DK / 64; ++x) {
                    tma_load_4d(t + L::KQ + x * 16384, &tk, 64 * x, c * C, hk, b, fb);
                    tma_load_4d(t + L::KQ + x * 16384 + 8192, &tq, 64 * x, c * C, hk, b, fb);
                }
                tma_load_4d(t + L::Y, &ty, col0, c * C, h, b, fb);
                tma_load_4d(t + L::Y + 8192, &ty, col0 + 64, c * C, h, b, fb);
                bulk_load(ring + L::G + (it % L::STAGES) * GATES, f.gates + cid * 3 * C, GATES, fb);
            };
            const int nblk = gridDim.x, blk = blockIdx.x;
            auto cid_of = [&](int it) { return chain * nc + chunks - 1 - it; };
            auto load_mats = [&](int it, int first, int n, int fb) {
                mbar_expect_tx(bar(fb), n * MAT);
                for (int m = first; m < first + n; ++m)
                    tma_load_2d(ring + L::N + m * MAT, &tm, 0, static_cast<int>((cid_of(it) * GDN_BACK_MATS + m) * C), bar(fb));
            };
            auto load_p = [&](int it) { load_mats(it, GDN_N_PARTS, GDN_BACK_MATS - GDN_N_PARTS, B_P); };
            auto load_n = [&](int it) { load_mats(it, 0, GDN_N_PARTS, B_N); };
            auto load_e = [&](int it) {
                mbar_expect_tx(bar(B_E), 32768);
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    tma_load_2d(ring + L::E + p * 16384, &te, 0, static_cast<int>(((cid_of(it) * 2 + p) * nblk + blk) * 128), bar(B_E));
            };
            int loaded = 0, np = 0, nn = 0, ne = 0;
            if (chunks > 0) {
                load(loaded++);
                load_p(np++);
                load_n(nn++);
                load_e(ne++);
                if (chunks > 1) load(loaded++);
            }
            for (int it = 0; it < chunks; ++it) {
                const uint32_t t = ring + (it % L::STAGES) * L::BYTES + L::Y;
                const int c = chunks - 1 - it;
                const bool more = it + 1 < chunks;
                const int64_t cid = cid_of(it);
                const int rs = static_cast<int>((cid * nblk + blk) * 128), rp = static_cast<int>((cid * 2 * nblk + blk) * 128);
                mbar_wait_or_dead(bar(B_KS), it & 1, dead);
                if (*dead) break;
#pragma unroll
                for (int x = 0; x < DK / 64; ++x) tma_store_2d(&tD, ring + L::KS + x * 16384, 64 * x, rs);
                bulk_commit();
                bulk_wait_read();
                mbar_arrive(bar(B_DFREE));
                mbar_wait_or_dead(bar(B_U), it & 1, dead);   // P, then N, then e are read: the next chunk's
                if (*dead) break;
                if (more) load_p(np++);
                mbar_wait_or_dead(bar(B_XN), it & 1, dead);
                if (*dead) break;
                if (more) load_n(nn++);
                mbar_wait_or_dead(bar(B_OUT), it & 1, dead); // d, and dv where the chunk's dy was
                if (*dead) break;
                if (more) load_e(ne++);
#pragma unroll
                for (int p = 0; p < 2; ++p) tma_store_2d(&td, ring + L::KS + p * 16384, 0, rp + p * nblk * 128);
                tma_store_4d(&tdv, t, col0, c * C, h, b);
                if (col0 + 64 < a.dv) tma_store_4d(&tdv, t + 8192, col0 + 64, c * C, h, b);
                bulk_commit();
                bulk_wait_read();
                mbar_arrive(bar(B_FREE));
                mbar_wait_or_dead(bar(B_UP), it & 1, dead);
                if (*dead) break;
                if (loaded < chunks) load(loaded++);
            }
            bulk_wait();
            if (*dead) {                                     // the copies in flight land before the CTA ends
                for (int j = loaded > L::STAGES ? loaded - L::STAGES : 0; j < loaded; ++j)
                    mbar_wait(bar(B_FULL + j % L::STAGES), (j / L::STAGES) & 1);
                if (np > 0) mbar_wait(bar(B_P), (np - 1) & 1);
                if (nn > 0) mbar_wait(bar(B_N), (nn - 1) & 1);
                if (ne > 0) mbar_wait(bar(B_E), (ne - 1) & 1);
            }
        }
    } else {
        regs_inc<BACK_REGS>();
        const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane, col = col0 + row;
        const int i0 = 32 * half;                            // this warp's tokens of a chunk
        const bool live = col < a.dv;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const int64_t per = static_cast<int64_t>(a.dk) * a.dv;
        constexpr int RD = DK / 2;                           // rows of d_k of a warp
        const uint32_t yat = L::Y + (row / 64) * 8192;
        float D[RD];
#pragma unroll
        for (int x = 0; x < RD; ++x) {
            const int rw = half * RD + x;
            D[x] = r.dstate != nullptr && live && rw < a.dk ? __ldcs(r.dstate + chain * per + static_cast<int64_t>(rw) * a.dv + col) : 0.f;
        }
        auto put_state = [&](int it) {                       // D after the chunk
            if (it > 0) mbar_wait_or_dead(bar(B_FREE), (it - 1) & 1, dead);
            __syncwarp();
#pragma unroll
            for (int x = 0; x < RD; x += 32) {
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = D[x + j];
                auto keep = [&](int j, const uint4& w) {     // 8 rows of d_k
                    const int at = half * RD + x + 8 * j;
                    *reinterpret_cast<uint4*>(ringp + L::KS + at / 64 * 16384 + box_at(row, at % 64 / 8)) = w;
                };
                put_part(lanes + d_at<DK>(0, half * RD + x), v, keep);
                put_part(lanes + d_at<DK>(1, half * RD + x), v);
                put_last(lanes + d_at<DK>(2, half * RD + x), v);
            }
            announce(bar(B_S), lane);
            hand_over(bar(B_KS), lane);
        };
        auto put_dy = [&](int it) {                          // dy and g dy of the chunk
            const int s = it % L::STAGES, n = len - (chunks - 1 - it) * C;
            const unsigned char* tile = ringp + s * L::BYTES;
            const float* gate = reinterpret_cast<const float*>(ringp + L::G + s * GATES);
            mbar_wait_or_dead(bar(B_FULL + s), (it / L::STAGES) & 1, dead);
            if (n < C) {                                     // K and Q rows past the length: zeros, whatever was there
                for (int p = tid; p < (C - n) * DK / 4; p += 32 * SW) {
                    const int e = p % 2, rw = n + (p / 2) / (DK / 8), x = (p / 2) % (DK / 8);
                    *reinterpret_cast<uint4*>(ringp + s * L::BYTES + L::KQ + (x / 8) * 16384 + e * 8192 + rw * 128 + (x % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async();
            }
            uint32_t y[16];
            float v[32];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int i = i0 + 2 * j;
                const uint32_t lo = *reinterpret_cast<const unsigned short*>(tile + yat + sw128_at(i, row % 64));
                const uint32_t hi = *reinterpret_cast<const unsigned short*>(tile + yat + sw128_at(i + 1, row % 64));
                y[j] = (i < n ? lo : 0u) | (i + 1 < n ? hi << 16 : 0u);
            }
            tmem_st16(lanes + Y_COL + i0 / 2, y);
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 g = *reinterpret_cast<const float4*>(gate + i0 + j);
                v[j] = a.scale * g.x * __uint_as_float(y[j / 2] << 16);
                v[j + 1] = a.scale * g.y * __uint_as_float(y[j / 2] & 0xffff0000u);
                v[j + 2] = a.scale * g.z * __uint_as_float(y[j / 2 + 1] << 16);
                v[j + 3] = a.scale * g.w * __uint_as_float(y[j / 2 + 1] & 0xffff0000u);
            }
            put_part(lanes + GY_COL + i0 / 2, v);
            put_part(lanes + GY_COL + 32 + i0 / 2, v);
            put_last(lanes + GY_COL + 64 + i0 / 2, v);
            __syncwarp();
            announce(bar(B_DY), lane);
        };
        if (chunks > 0) {
            put_dy(0);
            put_state(0);
        }
        for (int it = 0; it < chunks; ++it) {
            const int s = it % L::STAGES, c = chunks - 1 - it, n = len - c * C;
            const uint32_t ph = it & 1;
            unsigned char* tile = ringp + s * L::BYTES;
            const float* gate = reinterpret_cast<const float*>(ringp + L::G + s * GATES);
            float u[32], w[32], ke[32];                      // ke: D^T k_j, then times e_j
            await(bar(B_U), ph, dead);
            tmem_ld32(lanes + X_COL + i0, u);                // step 2
            tmem_ld32(lanes + Z_COL + i0, w);
            bar_pair(quad);                                  // beta x goes where this quarter's dy^T P was
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 h4 = *reinterpret_cast<const float4*>(gate + 2 * C + i0 + j), b4 = *reinterpret_cast<const float4*>(gate + C + i0 + j);
                const float hj[4] = {h4.x, h4.y, h4.z, h4.w}, bj[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ke[j + e] = u[j + e];
                    u[j + e] = fmaf(hj[e], u[j + e], a.scale * w[j + e]);
                    w[j + e] = bj[e] * u[j + e];
                }
            }
            put_part(lanes + Z_COL + i0 / 2, w);
            put_part(lanes + Z_COL + 32 + i0 / 2, w);
            put_last(lanes + Z3_COL + i0 / 2, w);
            announce(bar(B_X), lane);
            const float g63 = gate[C - 1];
            mbar_wait_or_dead(bar(B_E), ph, dead);
            const unsigned char* const ep = ringp + L::E;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float hi[8], lo[8];
                unpack16<BF16>(*reinterpret_cast<const uint4*>(ep + box_at(row, i0 / 8 + j)), hi);
                unpack16<BF16>(*reinterpret_cast<const uint4*>(ep + 16384 + box_at(row, i0 / 8 + j)), lo);
#pragma unroll
                for (int e = 0; e < 8; ++e) ke[8 * j + e] *= hi[e] + lo[e];
            }
            r.ke[(((chain * nc + c) * gridDim.x + blockIdx.x) * 4 + quad) * C + i0 + lane] = sum_lanes(ke, lane);
            await(bar(B_XN), ph, dead);
            tmem_ld32(lanes + X_COL + i0, w);                // step 4
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] += w[j];       // d
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 g4 = *reinterpret_cast<const float4*>(gate + i0 + j), b4 = *reinterpret_cast<const float4*>(gate + C + i0 + j);
                w[j] = -g4.x * (b4.x * u[j]);
                w[j + 1] = -g4.y * (b4.y * u[j + 1]);
                w[j + 2] = -g4.z * (b4.z * u[j + 2]);
                w[j + 3] = -g4.w * (b4.w * u[j + 3]);
            }
            put_part(lanes + S_COL + i0 / 2, w);
            put_part(lanes + S_COL + 32 + i0 / 2, w);
            put_last(lanes + S_COL + 64 + i0 / 2, w);
            announce(bar(B_H), lane);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const int i = i0 + j;
                *reinterpret_cast<__nv_bfloat16*>(tile + yat + sw128_at(i, row % 64)) = __float2bfloat16_rn(i < n ? gate[C + i] * u[j] : 0.f);
            }
            mbar_wait_or_dead(bar(B_DFREE), ph, dead);       // D has left the place
            __syncwarp();
            keep_parts(ringp + L::KS, row, i0 / 8, u);
            hand_over(bar(B_OUT), lane);
            if (it + 1 < chunks) put_dy(it + 1);
            await(bar(B_UP), ph, dead);
#pragma unroll
            for (int x = 0; x < RD; x += 32) {               // step 6
                float v[32];
                tmem_ld32(lanes + A_COL + half * RD + x, v);
#pragma unroll
                for (int j = 0; j < 32; ++j) D[x + j] = fmaf(g63, D[x + j], v[j]);
            }
            if (it + 1 < chunks) put_state(it + 1);
        }
        if (live) {
            if (r.dstate0 != nullptr) {
#pragma unroll
                for (int x = 0; x < RD; ++x) {
                    const int rw = half * RD + x;
                    if (rw < a.dk) __stcs(r.dstate0 + chain * per + static_cast<int64_t>(rw) * a.dv + col, D[x]);
                }
            }
            __nv_bfloat16* dv = static_cast<__nv_bfloat16*>(r.dv) + gdn_base(a.token_major, b, h, a.H, a.T, a.dv) + col;
            const int64_t vs = gdn_stride(a.token_major, a.H, a.dv);          // chunks past the length
            for (int t = chunks * C + half; t < a.T; t += 2) dv[t * vs] = __float2bfloat16_rn(0.f);
        }
    }
    tc_before_sync();
    __syncthreads();
    if (tid == 0 && ctl.dead) flag_error(a.err, ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, T_COLS);
}

template <int DK>
cudaError_t back(const CUtensorMap& tk, const CUtensorMap& tq, const CUtensorMap& ty, const CUtensorMap& tdv, const CUtensorMap& tm,
                 const CUtensorMap& tD, const CUtensorMap& td, const CUtensorMap& te, const GdnBack& r, const GdnFactors& f, cudaStream_t stream) {
    constexpr size_t smem = back_smem<DK>();
    static std::atomic<int> regs{0};
    cudaError_t e = check_kernel_registers(k_gdn_back<DK>, LAUNCH_REGS, regs);
    if (e != cudaSuccess) return e;
    static std::atomic<unsigned long long> seen;
    e = allow_smem(k_gdn_back<DK>, smem, seen);
    if (e != cudaSuccess) return e;
    k_gdn_back<DK><<<dim3((r.a.dv + 127) / 128, r.a.H, r.a.B), ST, smem, stream>>>(tk, tq, ty, tdv, tm, tD, td, te, r, f, (r.a.T + C - 1) / C);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_gdn_back(const GdnBack& r, const GdnFactors& f, cudaStream_t stream) {
    const GdnArgs& a = r.a;
    if (f.mats != GDN_BACK_MATS) return cudaErrorInvalidValue;
    const int64_t chunks = static_cast<int64_t>(a.B) * a.H * ((a.T + C - 1) / C);
    const int nblk = (a.dv + 127) / 128;
    CUtensorMap tk, tq, ty, tdv, tm, tD, td, te;
    if (!token_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk) || !token_map(&tq, a.q, a.token_major, a.B, a.Hk, a.T, a.dk) ||
        !token_map(&ty, r.dy, a.token_major, a.B, a.H, a.T, a.dv) || !token_map(&tdv, r.dv, a.token_major, a.B, a.H, a.T, a.dv) ||
        !row_map(&tm, f.mat, chunks * f.mats * C, C, C) || !row_map(&tD, r.keep_D, chunks * nblk * 128, a.dk <= 64 ? 64 : 128, 128) ||
        !row_map(&td, r.keep_d, chunks * 2 * nblk * 128, C, 128) || !row_map(&te, r.e, chunks * 2 * nblk * 128, C, 128))
        return cudaErrorInvalidValue;
    return a.dk <= 64 ? back<64>(tk, tq, ty, tdv, tm, tD, td, te, r, f, stream) : back<128>(tk, tq, ty, tdv, tm, tD, td, te, r, f, stream);
}

}  // namespace sdm
