// pc_wave.h -- sums over a wavefront and a workgroup by register exchanges
// between neighbouring lanes (DPP), without LDS for the wavefront's part: a
// step takes a few cycles where an exchange through LDS takes over a hundred.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcr {

// The value of the lane that the control names, 0 where there is none or the
// row of 16 lanes is not in the mask.
template <int kCtrl, int kRows>
__device__ __forceinline__ int32_t from_lane(int32_t x) {
    return __builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xf, false);
}
template <int kCtrl, int kRows>
__device__ __forceinline__ int64_t from_lane(int64_t x) {
    const uint32_t lo = (uint32_t)from_lane<kCtrl, kRows>((int32_t)x);
    const uint32_t hi = (uint32_t)from_lane<kCtrl, kRows>((int32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Sums over the lanes up to and with this one; all lanes take part.
template <typename N>
__device__ __forceinline__ N wave_scan(N x) {
    x += from_lane<0x111, 0xf>(x);      // 1, 2, 4, 8 lanes before, within rows of 16
    x += from_lane<0x112, 0xf>(x);
    x += from_lane<0x114, 0xf>(x);
    x += from_lane<0x118, 0xf>(x);
    x += from_lane<0x142, 0xa>(x);      // the last lane of the row before, in rows 1 and 3
    x += from_lane<0x143, 0xc>(x);      // lane 31, in rows 2 and 3
    return x;
}
__device__ __forceinline__ int32_t wave_last(int32_t x) { return __builtin_amdgcn_readlane(x, 63); }
__device__ __forceinline__ int64_t wave_last(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)wave_last((int32_t)(x >> 32)) << 32 | (uint32_t)wave_last((int32_t)x));
}

// Sums of K words over a workgroup's NT threads: exclusive ones in v, those
// over all in total.  lds: K * NT / 64 words.
template <int NT, int K, typename N>
__device__ __forceinline__ void block_scan(N (&v)[K], N (&total)[K], N *lds) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    N x[K];
#pragma unroll
    for (int i = 0; i < K; ++i) x[i] = wave_scan(v[i]);
    __syncthreads();
    if (lane == 63)
#pragma unroll
        for (int i = 0; i < K; ++i) lds[w * K + i] = x[i];
    __syncthreads();
    N t[NT / 64][K];
#pragma unroll
    for (int k = 0; k < NT / 64; ++k)
#pragma unroll
        for (int i = 0; i < K; ++i) t[k][i] = lds[k * K + i];
#pragma unroll
    for (int i = 0; i < K; ++i) {
        v[i] = x[i] - v[i];
        total[i] = 0;
#pragma unroll
        for (int k = 0; k < NT / 64; ++k) {
            v[i] += k < w ? t[k][i] : 0;
            total[i] += t[k][i];
        }
    }
}
template <int NT, typename N>
__device__ __forceinline__ N block_sum(N x, N *total, N *lds) {    // one word: its exclusive sum
    N v[1] = {x}, all[1];
    block_scan<NT>(v, all, lds);
    *total = all[0];
    return v[0];
}

}  // namespace pcr
