// What the tensor-core kernels of the gated delta rule share: tensor maps, operands as bf16 parts in
// TMEM, hand-over between warps.
#pragma once
#include "gdn_internal.h"
#include "tc_common.cuh"

namespace sdm {
namespace gdn {

using namespace tc;

constexpr int C = GDN_C64;
constexpr uint32_t MAT = C * C * 2;          // bytes of one [64][64] bf16 matrix
constexpr uint32_t GATES = 3 * C * 4;

// [B, heads, T, d] or [B, T, heads, d] bf16 as {d, T, heads, B}, boxes of 64 values x 64 tokens.
inline bool token_map(CUtensorMap* m, const void* base, int token_major, int B, int heads, int T, int d) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = map_encoder();
    if (!enc) return false;
    const cuuint64_t row = static_cast<cuuint64_t>(d) * 2, uT = T, uH = heads;
    cuuint64_t dim[4] = {static_cast<cuuint64_t>(d), uT, uH, static_cast<cuuint64_t>(B)};
    cuuint64_t str[3] = {token_major ? row * uH : row, token_major ? row : row * uT, row * uH * uT};
    cuuint32_t box[4] = {64, C, 1, 1}, es[4] = {1, 1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dim, str, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Row-major [rows][cols] bf16, boxes of 64 values x box_rows.
inline bool row_map(CUtensorMap* m, const void* base, int64_t rows, int cols, int box_rows) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = map_encoder();
    if (!enc) return false;
    cuuint64_t dim[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    cuuint64_t str[1] = {static_cast<cuuint64_t>(cols) * 2};
    cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)}, es[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dim, str, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The next bf16 part of 32 values into 16 packed columns (and to `keep`); the values keep what its rounding left.
struct KeepNone {
    __device__ __forceinline__ void operator()(int, const uint4&) const {}
};
template <class Keep = KeepNone>
__device__ __forceinline__ void put_part(uint32_t taddr, float (&v)[32], Keep keep = Keep{}) {
    uint32_t u[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) u[j] = split2(v[2 * j], v[2 * j + 1], v[2 * j], v[2 * j + 1]);
    tmem_st16(taddr, u);
#pragma unroll
    for (int j = 0; j < 4; ++j) keep(j, make_uint4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]));
}
// Where the 16-byte piece `piece` of row `row` lies in a swizzled box of 128-byte rows.
__device__ __forceinline__ uint32_t box_at(int row, int piece) { return row * 128 + ((piece ^ (row & 7)) << 4); }
// 32 values (pieces piece0 .. + 3 of the row) as two bf16 parts in two boxes of 128 rows, one after the other.
__device__ __forceinline__ void keep_parts(unsigned char* box, int row, int piece0, float (&v)[32]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t u[4], w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float& x = v[8 * j + 2 * e];
            float& y = v[8 * j + 2 * e + 1];
            u[e] = split2(x, y, x, y);
            w[e] = pack2(x, y);
        }
        unsigned char* const at = box + box_at(row, piece0 + j);
        *reinterpret_cast<uint4*>(at) = make_uint4(u[0], u[1], u[2], u[3]);
        *reinterpret_cast<uint4*>(at + 16384) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ void put_last(uint32_t taddr, const float (&v)[32]) {
    uint32_t u[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) u[j] = pack2(v[2 * j], v[2 * j + 1]);
    tmem_st16(taddr, u);
}
// 32 neighbouring floats of shared memory (16-byte aligned, the same for the whole warp).
__device__ __forceinline__ void get32(const float* p, float (&v)[32]) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float4 f = *reinterpret_cast<const float4*>(p + 4 * q);
        v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
    }
}
// Sums over the lanes of 32 values per lane: lane l gets the sum of value l.
__device__ __forceinline__ float sum_lanes(float (&v)[32], int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int j = 0; j < o; ++j) {
            const float give = up ? v[j] : v[j + o], keep = up ? v[j + o] : v[j];
            v[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    return v[0];
}

// A warp's share of an operand is in TMEM: tells the issuing warp.
__device__ __forceinline__ void announce(uint32_t bar, int lane) {
    tmem_st_wait();
    tc_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void await(uint32_t bar, uint32_t parity, volatile int* dead) {
    mbar_wait_or_dead(bar, parity, dead);
    __syncwarp();
    tc_after_sync();
}
// The same for what a warp has put into shared memory for the copies.
__device__ __forceinline__ void hand_over(uint32_t bar, int lane) {
    fence_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}
// Element (row, x) of a tile of 64-value, 128-byte rows, swizzled as TMA leaves it.
__device__ __forceinline__ uint32_t sw128_at(int row, int x) { return row * 128 + ((x * 2) ^ ((row & 7) << 4)); }

}  // namespace gdn
}  // namespace sdm
