// Shared by the kernels on the ragged cache of 8 bits.
#pragma once

#include "common.cuh"

namespace aircache {

constexpr int kScaleRows = AIRCACHE_SCALE_ROWS;

#ifdef __CUDACC__
// Rows in use of region r: lens[r], or none where its rows or blocks of scales would leave the buffers or the region.
__device__ __forceinline__ int rows_in_use(const int64_t *offsets, const int32_t *lens, int r, int64_t rows,
                                           int64_t first_region, int64_t scale_blocks) {
    const int64_t o = offsets[r], end = offsets[r + 1];
    const int n = lens[r];
    if (n <= 0 || o < 0 || end > rows || n > end - o) return 0;
    if (o / kScaleRows + first_region + r + (n + kScaleRows - 1) / kScaleRows > scale_blocks) return 0;
    return n;
}

// Two e4m3 codes (exact in fp16).
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
    return r;
}
__device__ __forceinline__ float2 e4m3x2_f32(uint32_t codes) {
    const uint32_t h = e4m3x2_f16x2(codes);
    float2 r;
    asm("{\n.reg .f16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}\n" : "=f"(r.x), "=f"(r.y) : "r"(h));
    return r;
}
#endif

}  // namespace aircache
