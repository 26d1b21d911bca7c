// Gated delta rule, gradients of q, k and the gates on the tensor cores (bf16 storage, d_k <= 128), every
// chunk of 64 tokens on its own, from what the two walks stored: the states S before and the gradients D
// after the chunks (transposed, bf16), e and d (transposed, two bf16 parts).  With the decay products G, g, h
// of a chunk, w = beta e and dy scaled:
//   dq_i = g_i S dy_i + sum_{j <= i} M_ij k_j,                           M_ij = G_ij beta_j <dy_i, e_j>
//   dk_j = beta_j h_j D e_j - beta_j g_j S d_j + sum_{i >= j} M_ij q_i
//          - sum_{i > j} A_ij k_i - sum_{i < j} A_ji k_i,                A_ij = beta_i beta_j G_ij <d_i, e_j>
//   dbeta_i = <d_i, e_i>
// and dalpha_t = sum_{j < t} (sum_{i >= t} prod_{t < l <= i} alpha_l X_ij) prod_{j < l < t} alpha_l over the
// gradients X of the decay products, with the chunk's start as column -1 and its end as row 64 (nothing is
// divided by a gate):
//   X_ij = beta_j <dy_i, e_j> q_i.k_j - beta_i beta_j <d_i, e_j> k_i.k_j,   X_{i,-1} = q_i.S dy_i - beta_i k_i.S d_i,
//   X_{64,j} = beta_j <D^T k_j, e_j>,   X_{64,-1} = <D, S>.
// The reverse walk has D^T k_j in fp32 and stores <D^T k_j, e_j>; from D as it is stored here, rounded to bf16, dalpha was off
// by 8e-3 at keys of a cosine of 0.98, along which D is small.
//
// One CTA per SM walks over the chunks of the key heads and adds up the value heads that share one.  The
// products over d_v have d_k as TMEM lanes (S and D are A operands as they lie), <dy, e> the tokens in
// lanes 0-63 and <d, e> in lanes 64-127, beside q.k and k.k.  Warps 0-7 take the products through registers,
// warp 8 issues the MMAs, warp 9 the copies, warps 10 and 11 run the sums of dalpha, a column a thread.
// The tiles of the next (head, block of d_v) load while this one's products are taken.  390 us at B = 8, H = 16, T = 4096,
// 128 x 128: 13,300 cycles a chunk and head, most of them the register stages (144 KB of tiles and 32 KB of Q and K would load
// in 7,400, the MMAs take 5,000); a third lane sum, in place of the walk's <D^T k_j, e_j>, cost 35 us more.
#include "gdn_tc.cuh"

#include <stddef.h>

namespace sdm {

namespace {

using namespace tc;
using namespace gdn;

constexpr int SW = 8, NT = 32 * (SW + 4);
constexpr int LAUNCH_REGS = 168, GRAD_REGS = 224, REST_REGS = 56;   // a thread's registers, at first and after the split
static_assert(GRAD_REGS >= LAUNCH_REGS && REST_REGS <= LAUNCH_REGS && SW * GRAD_REGS + 4 * REST_REGS <= (SW + 4) * LAUNCH_REGS, "register split");
// X below its diagonal, row by row: row i (0 .. 64) has columns -1 .. i - 1
__device__ __forceinline__ constexpr int x_at(int i, int col) { return i * (i + 1) / 2 + col; }      // column j: col = j + 1
// TMEM columns
constexpr uint32_t SY = 0, SD = 64, DE = 128, QK = 192, YE = 256, GE = 320, IQ = 384, IK = 448, T_COLS = 512;

template <int DK>
struct Tile {
    // per 64 values of d_k: 64 rows of Q, 64 of K.  M: M in two parts, -A; then dq and dk on their way to memory.  The d tile has 16 KB before it and the dy tile 8 KB after
    // it that the other half of the lanes of their products reads.
    static constexpr uint32_t QK = 0, S = 128 * 2 * DK, D = S + 256 * DK, E = D + 256 * DK, DT = E + 32768, Y = DT + 32768, M = Y + 16384,
                              G = M + 4 * MAT, BYTES = G + 1024;
    static constexpr uint32_t LOAD = 512 * DK + 65536 + 16384 + GATES;
};
enum { B_KQ = 0, B_TILE, B_INTER, B_INTRA, B_KREADY, B_M, B_READ, B_X, B_KFREE, B_OUT, B_XFREE, B_EMPTY, B_MFREE, B_COUNT };
struct Ctl {
    float X[(C + 1) * (C + 2) / 2];
    float dots[4][C];                          // X_{i,-1}, the share of each lane quarter
    alignas(16) float gt[3][C];                // g, beta, h of the head's chunk
    float db[C];
    float es[SW];
    uint4 al[C / 8];
    unsigned long long bar[B_COUNT];
    uint32_t tmem;
    int dead;
};
static_assert(offsetof(Ctl, gt) % 16 == 0 && offsetof(Ctl, al) % 16 == 0 && offsetof(Ctl, bar) % 8 == 0, "alignment of the wide reads");
template <int DK>
constexpr size_t grads_smem() { return 1024 + Tile<DK>::BYTES + sizeof(Ctl); }

__device__ __forceinline__ void bar_compute() { asm volatile("bar.sync 1, %0;\n" ::"n"(32 * SW) : "memory"); }

// A warp of which every lane has put something into shared memory for the MMAs or other warps.
__device__ __forceinline__ void arrive(uint32_t bar, int lane) {
    tc_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}

template <int DK>
__global__ void __launch_bounds__(NT, 1) k_gdn_grads_tc(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                                                        const __grid_constant__ CUtensorMap ty, const __grid_constant__ CUtensorMap tS,
                                                        const __grid_constant__ CUtensorMap tD, const __grid_constant__ CUtensorMap te,
                                                        const __grid_constant__ CUtensorMap td, const __grid_constant__ CUtensorMap tdq,
                                                        const __grid_constant__ CUtensorMap tdk, const GdnGradsTc r, int nc) {
    using L = Tile<DK>;
    extern __shared__ unsigned char raw[];
    const GdnArgs& a = r.a;
    const uint32_t base = smem_u32(raw);
    const uint32_t t = (base + 1023u) & ~1023u;
    unsigned char* const tp = raw + (t - base);
    Ctl& ctl = *reinterpret_cast<Ctl*>(tp + L::BYTES);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t bars = smem_u32(&ctl.bar[0]);
    auto bar = [&](int i) { return bars + 8 * i; };
    if (tid == 0) {
        ctl.dead = 0;
        for (int i = 0; i < B_COUNT; ++i) mbar_init(bar(i), i < B_KREADY ? 1 : i == B_XFREE ? 2 : i == B_EMPTY ? SW + 1 : i == B_MFREE ? 1 : SW);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
    }
    if (warp == 0) tmem_alloc(smem_u32(&ctl.tmem), T_COLS);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = ctl.tmem;
    volatile int* dead = &ctl.dead;
    const int group = a.H / a.Hk, nblk = (a.dv + 127) / 128, subs = group * nblk;
    const int64_t items = static_cast<int64_t>(a.B) * a.Hk * nc;
    // the chunks with tokens, in the order in which every warp of the CTA meets them
    struct Item {
        int b, hk, c, n;
    };
    auto item_of = [&](int64_t w) {
        Item x;
        x.c = static_cast<int>(w % nc);
        x.hk = static_cast<int>(w / nc % a.Hk);
        x.b = static_cast<int>(w / nc / a.Hk);
        const int left = gdn_length(a, x.b) - x.c * C;
        x.n = left < 0 ? 0 : left < C ? left : C;
        return x;
    };

    if (warp >= SW) {
        regs_dec<REST_REGS>();
    if (warp == SW) {                                        // MMAs
        const uint32_t id = mma_idesc(64), idA = id | MN_A, idB = id | MN_B, idAB = id | MN_A | MN_B;
        const uint64_t q = sw128_desc(t + L::QK), k = sw128_desc(t + L::QK + 8192), qt = sw128_mn_desc(t + L::QK, 16384),
                       kt = sw128_mn_desc(t + L::QK + 8192, 16384), S = sw128_mn_desc(t + L::S, 16384), D = sw128_mn_desc(t + L::D, 16384),
                       e = sw128_mn_desc(t + L::E, 8192), d = sw128_mn_desc(t + L::DT, 8192), dh = sw128_mn_desc(t + L::DT - 16384, 16384),
                       y = sw128_desc(t + L::Y), m = sw128_desc(t + L::M), mt = sw128_mn_desc(t + L::M, 8192);
        // rolled loops: unrolled, the descriptors of 80 MMAs are kept in registers and spilled
        uint32_t ni = 0, ns = 0, nh = 0;
        for (int64_t w = blockIdx.x; w < items; w += gridDim.x) {
            if (item_of(w).n == 0) continue;
            for (int sub = 0; sub < subs; ++sub, ++ns) {
                const uint32_t first = sub % nblk == 0 ? 0u : 1u;
                if (first == 0 && nh > 0) await(bar(B_READ), (nh - 1) & 1, dead);   // the last head's are taken
                await(bar(B_TILE), ns & 1, dead);
                if (elect_one()) {
#pragma unroll 1
                    for (int kk = 0; kk < 8; ++kk)           // S dy^T, <dy, e>
                        mma_bf16(tmem + SY, S + kk * 128, y + (kk / 4) * 512 + (kk % 4) * 2, idA, first | (kk != 0));
#pragma unroll 1
                    for (int p = 0; p < 2; ++p)
#pragma unroll 1
                        for (int kk = 0; kk < 8; ++kk) {
                            mma_bf16(tmem + SD, S + kk * 128, d + p * 1024 + kk * 128, idAB, first | (p | kk) != 0);
                            mma_bf16(tmem + DE, D + kk * 128, e + p * 1024 + kk * 128, idAB, first | (p | kk) != 0);
                            mma_bf16(tmem + YE, y + (kk / 4) * 512 + (kk % 4) * 2, e + p * 1024 + kk * 128, idB, first | (p | kk) != 0);
                        }
#pragma unroll 1
                    for (int p = 0; p < 3; ++p)              // <d, e>: (upper, upper), (upper, lower), (lower, upper)
#pragma unroll 1
                        for (int kk = 0; kk < 8; ++kk)
                            mma_bf16(tmem + GE, dh + (p == 2 ? 1024 : 0) + kk * 128, e + (p == 1 ? 1024 : 0) + kk * 128, idAB, first | (p | kk) != 0);
                    mma_commit(bar(B_EMPTY));
                }
                __syncwarp();
                if (sub == nblk - 1) {                       // first head: q.k and k.k, now that Q and K are there
                    await(bar(B_KQ), ni & 1, dead);
                    await(bar(B_KREADY), ni & 1, dead);
                    ++ni;
                    if (elect_one()) {
#pragma unroll 1
                        for (int kk = 0; kk < DK / 16; ++kk)
                            mma_bf16(tmem + QK, q + (kk / 4) * 1024 + (kk % 4) * 2, k + (kk / 4) * 1024 + (kk % 4) * 2, id, kk != 0);
                    }
                    __syncwarp();
                }
                if (sub % nblk == nblk - 1) {
                    if (elect_one()) mma_commit(bar(B_INTER));
                    __syncwarp();
                    await(bar(B_M), nh & 1, dead);
                    ++nh;
                    if (elect_one()) {
#pragma unroll 1
                        for (int p = 0; p < 2; ++p)
#pragma unroll 1
                            for (int kk = 0; kk < C / 16; ++kk) {
                                mma_bf16(tmem + IQ, kt + kk * 128, m + p * (MAT / 16) + kk * 2, idA, (p | kk) != 0);
                                mma_bf16(tmem + IK, qt + kk * 128, mt + p * (MAT / 16) + kk * 128, idAB, (p | kk) != 0);
                            }
#pragma unroll 1
                        for (int kk = 0; kk < C / 16; ++kk) {
                            mma_bf16(tmem + IK, kt + kk * 128, mt + 2 * (MAT / 16) + kk * 128, idAB, 1);
                            mma_bf16(tmem + IK, kt + kk * 128, m + 2 * (MAT / 16) + kk * 2, idA, 1);
                        }
                        mma_commit(bar(B_INTRA));
                    }
                    __syncwarp();
                }
            }
        }
    } else if (warp == SW + 1) {                             // copies
        if (lane == 0) {
            uint32_t ni = 0, ns = 0;
            Item last{0, 0, 0, 0};                           // whose dq and dk are still to be stored
            auto store = [&]() {                             // they lie where M and A were
                mbar_wait_or_dead(bar(B_OUT), (ni - 1) & 1, dead);
                if (*dead) return;
#pragma unroll
                for (int i = 0; i < DK / 64; ++i) {
                    if (64 * i < a.dk) {
                        tma_store_4d(&tdq, t + L::M + i * 8192, 64 * i, last.c * C, last.hk, last.b);
                        tma_store_4d(&tdk, t + L::M + 16384 + i * 8192, 64 * i, last.c * C, last.hk, last.b);
                    }
                }
                bulk_commit();
                bulk_wait_read();
                mbar_arrive(bar(B_MFREE));
            };
            for (int64_t w = blockIdx.x; w < items && !*dead; w += gridDim.x) {
                const Item x = item_of(w);
                if (x.n == 0) continue;
                for (int sub = 0; sub < subs; ++sub, ++ns) {
                    const int h = x.hk * group + sub / nblk, blk = sub % nblk;
                    const int64_t cid = (static_cast<int64_t>(x.b) * a.H + h) * nc + x.c;
                    const int rs = static_cast<int>((cid * nblk + blk) * 128), rp = static_cast<int>((cid * 2 * nblk + blk) * 128);
                    if (ns > 0) {
                        mbar_wait_or_dead(bar(B_EMPTY), (ns - 1) & 1, dead);
                        if (*dead) break;
                    }
                    mbar_expect_tx(bar(B_TILE), L::LOAD);
#pragma unroll
                    for (int i = 0; i < DK / 64; ++i) tma_load_2d(t + L::S + i * 16384, &tS, 64 * i, rs, bar(B_TILE));
                    tma_load_4d(t + L::Y, &ty, blk * 128, x.c * C, h, x.b, bar(B_TILE));
                    tma_load_4d(t + L::Y + 8192, &ty, blk * 128 + 64, x.c * C, h, x.b, bar(B_TILE));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        tma_load_2d(t + L::E + i * 16384, &te, 0, rp + i * nblk * 128, bar(B_TILE));
                        tma_load_2d(t + L::DT + i * 16384, &td, 0, rp + i * nblk * 128, bar(B_TILE));
                    }
#pragma unroll
                    for (int i = 0; i < DK / 64; ++i) tma_load_2d(t + L::D + i * 16384, &tD, 64 * i, rs, bar(B_TILE));
                    bulk_load(t + L::G, r.gates + cid * 3 * C, GATES, bar(B_TILE));
                    if (sub == 0) {                          // Q and K, once the last chunk's are done with
                        if (ni > 0) mbar_wait_or_dead(bar(B_KFREE), (ni - 1) & 1, dead);
                        mbar_expect_tx(bar(B_KQ), 256 * DK);
#pragma unroll
                        for (int i = 0; i < DK / 64; ++i) {
                            tma_load_4d(t + L::QK + i * 16384, &tq, 64 * i, x.c * C, x.hk, x.b, bar(B_KQ));
                            tma_load_4d(t + L::QK + i * 16384 + 8192, &tk, 64 * i, x.c * C, x.hk, x.b, bar(B_KQ));
                        }
                        if (ni > 0) store();
                        last = x;
                        ++ni;
                    }
                }
            }
            if (ni > 0 && !*dead) store();
            bulk_wait();
            if (*dead) {                                     // the copies in flight land before the CTA ends
                if (ns > 0) mbar_wait(bar(B_TILE), (ns - 1) & 1);
                if (ni > 0) mbar_wait(bar(B_KQ), (ni - 1) & 1);
            }
        }
    } else if (warp > SW + 1) {                              // dalpha, dbeta: column j = tj - 1, then token tj
        const int tj = tid - 32 * (SW + 2);
        uint32_t nh = 0;
        for (int64_t w = blockIdx.x; w < items; w += gridDim.x) {
            const Item x = item_of(w);
            const int t0 = x.c * C, nt = a.T - t0 < C ? a.T - t0 : C;
            for (int hv = 0; hv < group; ++hv) {
                const int64_t at = (static_cast<int64_t>(x.b) * a.H + x.hk * group + hv) * a.T + t0 + tj;
                float s = 0.f, db = 0.f;
                if (x.n > 0) {
                    mbar_wait_or_dead(bar(B_X), nh & 1, dead);
                    ++nh;
                    // blocks of eight rows, read before any of them is written: the loads do not wait for each other
                    float acc = ctl.X[x_at(C, tj)], next = 1.f;              // the end's row; alpha of the row below
#pragma unroll 1
                    for (int q8 = C / 8 - 1; q8 >= tj / 8; --q8) {
                        float al[8], v[8];
                        unpack16<BF16>(ctl.al[q8], al);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = 8 * q8 + e >= tj ? ctl.X[x_at(8 * q8 + e, tj)] : 0.f;
#pragma unroll
                        for (int e = 7; e >= 0; --e) {
                            acc = fmaf(next, acc, v[e]);
                            next = al[e];
                            if (8 * q8 + e >= tj) ctl.X[x_at(8 * q8 + e, tj)] = acc;
                        }
                    }
                    float p = 1.f;
#pragma unroll 1
                    for (int q8 = tj / 8; q8 < C / 8; ++q8) {
                        float al[8], v[8];
                        unpack16<BF16>(ctl.al[q8], al);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = 8 * q8 + e >= tj ? ctl.X[x_at(8 * q8 + e, tj)] : 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            if (8 * q8 + e >= tj) {
                                ctl.X[x_at(8 * q8 + e, tj)] = v[e] * p;
                                p *= al[e];
                            }
                        }
                    }
                    asm volatile("bar.sync 2, 64;\n" ::: "memory");
#pragma unroll 8
                    for (int i = 0; i < C; ++i) s += i <= tj ? ctl.X[x_at(tj, i)] : 0.f;
                    db = ctl.db[tj];
                    arrive(bar(B_XFREE), lane);
                }
                if (tj < nt) {
                    static_cast<__nv_bfloat16*>(r.dalpha)[at] = __float2bfloat16_rn(tj < x.n ? s : 0.f);
                    static_cast<__nv_bfloat16*>(r.dbeta)[at] = __float2bfloat16_rn(tj < x.n ? db : 0.f);
                }
            }
        }
    }
    } else {
        regs_inc<GRAD_REGS>();
        const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane, i0 = 32 * half;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const float* gate = reinterpret_cast<const float*>(tp + L::G);
        const unsigned char* kq = tp + L::QK + (row / 64) * 16384;   // this lane's column of Q; K 8192 bytes on
        const int i = row & 63;                              // token of this lane in <dy, e> and <d, e>
        uint32_t ni = 0, ns = 0, nh = 0;
        for (int64_t w = blockIdx.x; w < items; w += gridDim.x) {
            const Item x = item_of(w);
            const int t0 = x.c * C, n = x.n, nt = a.T - t0 < C ? a.T - t0 : C;
            if (n == 0) {                                    // past the length
                const int64_t at = gdn_base(a.token_major, x.b, x.hk, a.Hk, a.T, a.dk), ks = gdn_stride(a.token_major, a.Hk, a.dk);
                for (int p = tid; p < nt * (a.dk / 8); p += 32 * SW) {
                    const int64_t o = at + (t0 + p / (a.dk / 8)) * ks + (p % (a.dk / 8)) * 8;
                    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(r.dq) + o) = make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(r.dk) + o) = make_uint4(0, 0, 0, 0);
                }
                continue;
            }
            float dq[32], dk[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) dq[j] = dk[j] = 0.f;
            for (int hv = 0; hv < group; ++hv, ++nh) {
                const int64_t chain = static_cast<int64_t>(x.b) * a.H + x.hk * group + hv;
                unsigned short al = 0x3f80;
                if (tid < n) al = __ldg(static_cast<const unsigned short*>(a.alpha) + chain * a.T + t0 + tid);
                float es = 0.f, gv = 0.f, ke = 0.f;          // <D, S>; a gate product of the head; <D^T k_j, e_j>
                if (tid < C) {
                    const float* at = r.ke + (chain * nc + x.c) * nblk * 4 * C + tid;
                    for (int p = 0; p < 4 * nblk; ++p) ke += __ldg(at + p * C);
                }
                for (int blk = 0; blk < nblk; ++blk, ++ns) {
                    mbar_wait_or_dead(bar(B_TILE), ns & 1, dead);
                    for (int p = tid; p < 16 * DK; p += 32 * SW) {
                        float u[8], v[8];
                        unpack16<BF16>(*reinterpret_cast<const uint4*>(tp + L::S + p * 16), u);
                        unpack16<BF16>(*reinterpret_cast<const uint4*>(tp + L::D + p * 16), v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) es = fmaf(u[e], v[e], es);
                    }
                    if (tid < 3 * C) gv = gate[tid];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(B_EMPTY));
                }
                if (hv == 0) {
                    mbar_wait_or_dead(bar(B_KQ), ni & 1, dead);
                    ++ni;
                    if (n < C) {                             // rows past the length: zeros, whatever was there
                        for (int p = tid; p < (C - n) * DK / 4; p += 32 * SW) {
                            const int e = p % 2, rw = n + (p / 2) / (DK / 8), c = (p / 2) % (DK / 8);
                            *reinterpret_cast<uint4*>(tp + L::QK + (c / 8) * 16384 + e * 8192 + rw * 128 + (c % 8) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_async();
                    }
                    arrive(bar(B_KREADY), lane);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) es += __shfl_xor_sync(0xffffffffu, es, o);
                if (nh > 0) mbar_wait_or_dead(bar(B_XFREE), (nh - 1) & 1, dead);
                // from here on nothing of the last head is read any more
                if (lane == 0) ctl.es[warp] = es;
                if (tid < 3 * C) (&ctl.gt[0][0])[tid] = gv;
                if (tid < C) reinterpret_cast<unsigned short*>(ctl.al)[tid] = al;
                bar_compute();
                if (hv == 0 && ni > 1) mbar_wait_or_dead(bar(B_MFREE), ni & 1, dead);   // the last outputs have left M's place
                await(bar(B_INTER), nh & 1, dead);
                {   // M (lanes 0-63) and -A (lanes 64-127), 32 columns of token i; their share of X
                    const bool isq = quad < 2;
                    float u[32], v[32];
                    tmem_ld32(lanes + (isq ? YE : GE) + i0, u);
                    tmem_ld32(lanes + QK + i0, v);
                    if (!isq && (i >> 5) == half) {
                        float diag = 0.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) diag = (i & 31) == j ? u[j] : diag;
                        ctl.db[i] = diag;
                    }
                    if ((quad & 1) == 0 && half == 1) {      // tokens 0-31 have no columns 32-63
#pragma unroll
                        for (int j = 0; j < 32; ++j) u[j] = v[j] = 0.f;
                    } else {
                        float G = 0.f;
                        if ((quad & 1) == 1 && half == 0) {  // from the diagonal down to column 32
#pragma unroll
                            for (int q8 = 7; q8 >= 4; --q8) {
                                float f[8];
                                unpack16<BF16>(ctl.al[q8], f);
#pragma unroll
                                for (int e = 7; e >= 0; --e) G = (8 * q8 + e == i ? 1.f : G) * f[e];
                            }
                        }
                        const float bi = i < n ? (isq ? a.scale : -ctl.gt[1][i]) : 0.f;
                        const int last = isq ? i : i - 1;
#pragma unroll
                        for (int q8 = 3; q8 >= 0; --q8) {
                            float f[8];
                            unpack16<BF16>(ctl.al[i0 / 8 + q8], f);
                            const float4 b0 = *reinterpret_cast<const float4*>(&ctl.gt[1][i0 + 8 * q8]), b1 = *reinterpret_cast<const float4*>(&ctl.gt[1][i0 + 8 * q8 + 4]);
                            const float be[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
#pragma unroll
                            for (int e = 7; e >= 0; --e) {
                                const int jj = 8 * q8 + e, j = i0 + jj;
                                G = j == i ? 1.f : G;
                                const float c = j <= last && i < n ? bi * (be[e] * u[jj]) : 0.f;
                                v[jj] *= c;                  // X
                                u[jj] = G * c;               // M, or -A
                                G *= f[e];
                            }
                        }
                    }
                    unsigned char* const mp = tp + L::M + (isq ? 0 : 2 * MAT) + i * 128;
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float& x0 = u[8 * q4 + 2 * e];
                            float& x1 = u[8 * q4 + 2 * e + 1];
                            hi[e] = split2(x0, x1, x0, x1);
                            lo[e] = pack2(x0, x1);
                        }
                        const uint32_t at = static_cast<uint32_t>(i0 / 8 + q4) ^ (i & 7);
                        *reinterpret_cast<uint4*>(mp + at * 16) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        if (isq) *reinterpret_cast<uint4*>(mp + MAT + at * 16) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    }
                    if (isq) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (i0 + j < i) ctl.X[x_at(i, i0 + j + 1)] = v[j];
                    }
                    fence_async();
                    arrive(bar(B_M), lane);
                    // the products over d_v: lanes are rows of d_k (the lanes past them are left out), columns tokens
                    const bool in = DK == 128 || row < DK;
                    uint32_t qc[16], kc[16];                 // this lane's q and k, two tokens in a word
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const unsigned char* x0 = kq + sw128_at(i0 + 2 * j, row % 64);
                        const unsigned char* x1 = kq + sw128_at(i0 + 2 * j + 1, row % 64);
                        qc[j] = *reinterpret_cast<const unsigned short*>(x0) | (static_cast<uint32_t>(*reinterpret_cast<const unsigned short*>(x1)) << 16);
                        kc[j] = *reinterpret_cast<const unsigned short*>(x0 + 8192) | (static_cast<uint32_t>(*reinterpret_cast<const unsigned short*>(x1 + 8192)) << 16);
                        if (!in) qc[j] = kc[j] = 0u;
                    }
                    auto at16 = [](const uint32_t (&w)[16], int j) { return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); };
                    // tokens past the length, and lanes past d_k, hold whatever was in the tiles
                    auto only = [&](float (&p)[32]) {
                        if (n < C || !in) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) p[j] = in && i0 + j < n ? p[j] : 0.f;
                        }
                    };
                    {
                        float p[32], c[32];
                        tmem_ld32(lanes + SY + i0, p);
                        only(p);
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 g = *reinterpret_cast<const float4*>(&ctl.gt[0][i0 + j]);
                            const float gj[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float x = a.scale * p[j + e];
                                dq[j + e] = fmaf(gj[e], x, dq[j + e]);
                                c[j + e] = x * at16(qc, j + e);
                            }
                        }
                        tmem_ld32(lanes + SD + i0, p);
                        only(p);
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 g = *reinterpret_cast<const float4*>(&ctl.gt[0][i0 + j]), b4 = *reinterpret_cast<const float4*>(&ctl.gt[1][i0 + j]);
                            const float gj[4] = {g.x, g.y, g.z, g.w}, bj[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float x = -bj[e] * p[j + e];
                                dk[j + e] = fmaf(gj[e], x, dk[j + e]);
                                c[j + e] = fmaf(x, at16(kc, j + e), c[j + e]);
                            }
                        }
                        ctl.dots[quad][i0 + lane] = sum_lanes(c, lane);
                        tmem_ld32(lanes + DE + i0, p);
                        only(p);
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 h4 = *reinterpret_cast<const float4*>(&ctl.gt[2][i0 + j]), b4 = *reinterpret_cast<const float4*>(&ctl.gt[1][i0 + j]);
                            const float hj[4] = {h4.x, h4.y, h4.z, h4.w}, bj[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) dk[j + e] = fmaf(hj[e], bj[e] * p[j + e], dk[j + e]);
                        }
                    }
                    arrive(bar(B_READ), lane);
                    bar_compute();
                    if (!isq) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (i0 + j < i) ctl.X[x_at(i, i0 + j + 1)] += v[j];
                    }
                    if (tid < C) {
                        ctl.X[x_at(tid, 0)] = (ctl.dots[0][tid] + ctl.dots[1][tid]) + (ctl.dots[2][tid] + ctl.dots[3][tid]);
                        ctl.X[x_at(C, tid + 1)] = ctl.gt[1][tid] * ke;
                        if (tid == 0) {
                            float e = 0.f;
                            for (int wp = 0; wp < SW; ++wp) e += ctl.es[wp];
                            ctl.X[x_at(C, 0)] = e;
                        }
                    }
                    arrive(bar(B_X), lane);
                    await(bar(B_INTRA), nh & 1, dead);
                    if (hv == group - 1) arrive(bar(B_KFREE), lane);         // q and k are done with
                    tmem_ld32(lanes + IQ + i0, u);
                    tmem_ld32(lanes + IK + i0, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        dq[j] += u[j];
                        dk[j] += v[j];
                    }
                }
            }
            if (row < DK) {
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    unsigned char* const to = tp + L::M + (row / 64) * 8192 + sw128_at(i0 + j, row % 64);
                    *reinterpret_cast<__nv_bfloat16*>(to) = __float2bfloat16_rn(i0 + j < n ? dq[j] : 0.f);
                    *reinterpret_cast<__nv_bfloat16*>(to + 16384) = __float2bfloat16_rn(i0 + j < n ? dk[j] : 0.f);
                }
            }
            fence_async();
            arrive(bar(B_OUT), lane);
        }
    }
    tc_before_sync();
    __syncthreads();
    if (tid == 0 && ctl.dead) flag_error(a.err, ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, T_COLS);
}

template <int DK>
cudaError_t grads(const GdnGradsTc& r, cudaStream_t stream) {
    const GdnArgs& a = r.a;
    const int nc = (a.T + C - 1) / C, nblk = (a.dv + 127) / 128;
    const int64_t chunks = static_cast<int64_t>(a.B) * a.H * nc, items = static_cast<int64_t>(a.B) * a.Hk * nc;
    CUtensorMap tq, tk, ty, tS, tD, te, td, tdq, tdk;
    if (!token_map(&tq, a.q, a.token_major, a.B, a.Hk, a.T, a.dk) || !token_map(&tk, a.k, a.token_major, a.B, a.Hk, a.T, a.dk) ||
        !token_map(&ty, r.dy, a.token_major, a.B, a.H, a.T, a.dv) || !row_map(&tS, r.S, chunks * nblk * 128, DK, 128) ||
        !row_map(&tD, r.D, chunks * nblk * 128, DK, 128) || !row_map(&te, r.e, chunks * 2 * nblk * 128, C, 128) ||
        !row_map(&td, r.d, chunks * 2 * nblk * 128, C, 128) || !token_map(&tdq, r.dq, a.token_major, a.B, a.Hk, a.T, a.dk) ||
        !token_map(&tdk, r.dk, a.token_major, a.B, a.Hk, a.T, a.dk))
        return cudaErrorInvalidValue;
    constexpr size_t smem = grads_smem<DK>();
    static std::atomic<int> regs{0};
    cudaError_t e = check_kernel_registers(k_gdn_grads_tc<DK>, LAUNCH_REGS, regs);
    if (e != cudaSuccess) return e;
    static std::atomic<unsigned long long> seen;
    e = allow_smem(k_gdn_grads_tc<DK>, smem, seen);
    if (e != cudaSuccess) return e;
    k_gdn_grads_tc<DK><<<static_cast<unsigned>(items < 152 ? items : 152), NT, smem, stream>>>(tq, tk, ty, tS, tD, te, td, tdq, tdk, r, nc);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_gdn_grads_tc(const GdnGradsTc& r, cudaStream_t stream) {
    return r.a.dk <= 64 ? grads<64>(r, stream) : grads<128>(r, stream);
}

}  // namespace sdm
