// Pieces the attention kernels share: the LDS layout of K and V rows, the order in which
// items go to the XCDs, and exchanges between the halves of a wave.
#pragma once

#include "device_common.h"

namespace rag {

__device__ __forceinline__ u32x4 ld16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }

// Element offset of (row, col) in [rows][64 channels] LDS storage (128-byte rows,
// two per 256-byte bank line) whose 16-byte chunks are XOR-swizzled by row bits
// 1-3: the K-operand reads (16 consecutive rows, one chunk each) then meet 16
// distinct bank groups, and in the transposed V reads (rows r..r+3, four
// adjacent chunks each) rows r and r+2 use opposite halves of the row.
__device__ __forceinline__ int kv_swz(int row) { return (((row >> 1) & 1) << 2) | ((row >> 2) & 3); }
__device__ __forceinline__ int kv_off(int row, int col) { return row * kHeadDim + ((((col >> 3) ^ kv_swz(row)) & 7) << 3) + (col & 7); }

constexpr float kSumCap = 65536.f;  // largest lane sum of a chunk's exponentials kept (2^16)
constexpr int kStreamRun = 8;

__device__ __forceinline__ int stream_item(int bid, int nb) {  // nb: a multiple of 8 * kStreamRun
    const int xcd = bid % 8, j = bid / 8;
    return ((j / kStreamRun) * 8 + xcd) * kStreamRun + j % kStreamRun;
}

__device__ __forceinline__ void attn_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The magnitude of the factor that makes powers of two of scores.  A factor of zero would turn hidden keys' -inf
// into NaN; the smallest fp32 value in its place leaves every exponential 1: times the largest score it is 5e-7.
__device__ __forceinline__ float softmax_factor(float scale) {
    return scale == 0.f ? 0x1p-149f : fabsf(scale) * 1.4426950408889634f;
}

// Combine a value with the one held by the lane 32 apart (the other half of
// the same query row): v_permlane32_swap hands each half the other's value.
__device__ __forceinline__ float max_xor32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float sum_xor32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace rag
