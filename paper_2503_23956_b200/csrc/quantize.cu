// aircache_quantize and aircache_append_quantized: the ragged cache in 8 bits.
//
// 64 rows of a region and one KV head share a scale, the smallest power of two s with max |x| <= 448 s (448 = the largest
// e4m3 number).  e4m3 is a floating-point type, so a scale between the powers of two would gain nothing but range; with
// a power of two x / s and code * s are exact, and a block whose scale grows keeps its numbers but for those that
// leave the normal range.
//
// Bound by memory: 2 bytes in and 1 out per element.  A block of 128 threads holds 64 rows of one head of K or V in
// registers (16 KB at 128 channels), all loads under way at once, takes the largest magnitude of the 16-bit patterns as
// integers, and stores the codes; heads and K / V of the same rows are neighbours in the grid, so that whole rows are
// read at about the same time.
#include "common.cuh"
#include "ptx.cuh"
#include "quantize.cuh"

namespace aircache {

namespace {

struct QuantizeParams {
    const char *k, *v;
    char *k8, *v8;
    float *k_scale, *v_scale;
    const int64_t *offsets;
    const int32_t *lens;
    int64_t rows, scale_blocks, first_region;
    int n_regions, heads;
};

// The exponent of a block's scale from its largest magnitude, a finite bf16 pattern without the sign: 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(uint32_t top) {
    const int e = (int)(top >> 7) - 127 - 8 + ((top & 0x7f) > 0x60 ? 1 : 0);
    return max(e, -126);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126..127

// Codes of two values; beyond 448 the largest number, NaN stays.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t magnitude) { return magnitude < 0x7f80 ? magnitude : 0; }

template <int D>
__global__ void __launch_bounds__(128) quantize_kernel(QuantizeParams p) {
    constexpr int LPR = D / 16;              // lanes of a row: 16 channels each
    constexpr int RPP = 128 / LPR;           // rows of a pass
    constexpr int PASSES = kScaleRows / RPP;
    __shared__ uint32_t s_top[4];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int which = blockIdx.x % (2 * p.heads), head = which >> 1;
    const int64_t b = blockIdx.x / (2 * p.heads);   // block of the call: block j of region r is offsets[r] / 64 - offsets[0] / 64 + r + j
    const int64_t b0 = p.offsets[0] / kScaleRows;
    int lo = 0, hi = p.n_regions;                    // the last region whose first block is at or before b
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const bool before = at < hi && p.offsets[at] / kScaleRows - b0 + at <= b;
        lo += (max(__popc(__ballot_sync(0xffffffffu, before)), 1) - 1) * step;
        hi = min(hi, lo + step);
    }
    const int r = lo;
    const int64_t o = p.offsets[r];
    const int n = rows_in_use(p.offsets, p.lens, r, p.rows, p.first_region, p.scale_blocks);
    const int64_t j = b - (o / kScaleRows - b0 + r);
    if (j < 0 || j * kScaleRows >= n) return;
    const int rows = min(kScaleRows, n - (int)j * kScaleRows);
    const int64_t row0 = o + j * kScaleRows;
    const char *src = (which & 1 ? p.v : p.k);
    char *dst = (which & 1 ? p.v8 : p.k8);
    const int row = threadIdx.x / LPR, c0 = threadIdx.x % LPR * 16;
    uint4 x[PASSES][2];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int at = row + i * RPP;
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        if (at < rows) {
            const char *from = src + (((row0 + at) * p.heads + head) * D + c0) * 2;
            x[i][0] = __ldcs(reinterpret_cast<const uint4 *>(from));
            x[i][1] = __ldcs(reinterpret_cast<const uint4 *>(from) + 1);
        }
    }
    uint32_t top2 = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            top2 = __vmaxu2(top2, x[i][h].x & 0x7fff7fffu);
            top2 = __vmaxu2(top2, x[i][h].y & 0x7fff7fffu);
            top2 = __vmaxu2(top2, x[i][h].z & 0x7fff7fffu);
            top2 = __vmaxu2(top2, x[i][h].w & 0x7fff7fffu);
        }
    uint32_t top = max(top2 & 0xffffu, top2 >> 16);
    if (top >= 0x7f80) {   // infinities and NaN do not count
        top = 0;
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w[4] = {x[i][h].x, x[i][h].y, x[i][h].z, x[i][h].w};
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    top = max(top, max(finite_or_zero(w[a] & 0x7fffu), finite_or_zero(w[a] >> 16 & 0x7fffu)));
            }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
    const int e = scale_exponent(max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3])));
    const float inv = power_of_two(-e);
    if (threadIdx.x == 0)
        (which & 1 ? p.v_scale : p.k_scale)[(o / kScaleRows + p.first_region + r + j) * p.heads + head] = power_of_two(e);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int at = row + i * RPP;
        uint32_t out[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w[4] = {x[i][h].x, x[i][h].y, x[i][h].z, x[i][h].w};
#pragma unroll
            for (int a = 0; a < 4; a += 2)
                out[2 * h + a / 2] = e4m3x2(bf16lo(w[a]) * inv, bf16hi(w[a]) * inv) |
                                     e4m3x2(bf16lo(w[a + 1]) * inv, bf16hi(w[a + 1]) * inv) << 16;
        }
        if (at < rows)
            *reinterpret_cast<uint4 *>(dst + ((row0 + at) * p.heads + head) * D + c0) = make_uint4(out[0], out[1], out[2], out[3]);
    }
}

// One block per region, one warp per (head, K or V): lens[r] is read by all of them before one adds to it.
template <int D>
__global__ void append_quantized_kernel(QuantizeParams p, int32_t *lens, const char *k_new, const char *v_new) {
    constexpr int CPL = D / 32;   // channels of a lane: 4 or 2
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int r = blockIdx.x, lane = threadIdx.x & 31, which = threadIdx.x >> 5, head = which >> 1;
    const int64_t o = p.offsets[r];
    const int n = lens[r];
    const bool room = n >= 0 && o >= 0 && o + n < p.offsets[r + 1] && o + n < p.rows &&
                      o / kScaleRows + p.first_region + r + n / kScaleRows < p.scale_blocks;
    __syncthreads();
    if (!room) return;
    if (threadIdx.x == 0) lens[r] = n + 1;
    const char *src = (which & 1 ? v_new : k_new) + (((int64_t)r * p.heads + head) * D + lane * CPL) * 2;
    uint32_t w[2] = {0, 0};
    if (CPL == 4) {
        const uint2 x = *reinterpret_cast<const uint2 *>(src);
        w[0] = x.x;
        w[1] = x.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t *>(src);
    }
    float *scale = (which & 1 ? p.v_scale : p.k_scale) +
                   (o / kScaleRows + p.first_region + r + n / kScaleRows) * p.heads + head;
    const int place = n % kScaleRows;
    const float held = *scale;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < CPL / 2; ++i)
        top = max(top, max(finite_or_zero(w[i] & 0x7fffu), finite_or_zero(w[i] >> 16 & 0x7fffu)));
    const int e = scale_exponent(__reduce_max_sync(0xffffffffu, top));
    float now = power_of_two(e), inv = power_of_two(-e);
    char *block = (which & 1 ? p.v8 : p.k8) + ((o + n - place) * p.heads + head) * D + lane * CPL;
    const int64_t pitch = (int64_t)p.heads * D;
    if (place > 0 && held >= now) {
        now = held;
        inv = 1.f / held;   // exact: a power of two
    } else if (place > 0) {
        const float shrink = held * inv;
#pragma unroll 4
        for (int i = 0; i < place; ++i) {
            char *at = block + i * pitch;
            if (CPL == 4) {
                const uint32_t x = *reinterpret_cast<const uint32_t *>(at);
                const float2 a = e4m3x2_f32(x & 0xffffu), b = e4m3x2_f32(x >> 16);
                *reinterpret_cast<uint32_t *>(at) = e4m3x2(a.x * shrink, a.y * shrink) | e4m3x2(b.x * shrink, b.y * shrink) << 16;
            } else {
                const float2 a = e4m3x2_f32(*reinterpret_cast<const uint16_t *>(at));
                *reinterpret_cast<uint16_t *>(at) = (uint16_t)e4m3x2(a.x * shrink, a.y * shrink);
            }
        }
    }
    char *at = block + place * pitch;
    const uint32_t first = e4m3x2(bf16lo(w[0]) * inv, bf16hi(w[0]) * inv);
    if (CPL == 4)
        *reinterpret_cast<uint32_t *>(at) = first | e4m3x2(bf16lo(w[1]) * inv, bf16hi(w[1]) * inv) << 16;
    else
        *reinterpret_cast<uint16_t *>(at) = (uint16_t)first;
    if (lane == 0) *scale = now;
}

QuantizeParams params_of(const aircache_shape_t *s, const aircache_quantized_t *c) {
    QuantizeParams p = {};
    p.k8 = static_cast<char *>(c->k);
    p.v8 = static_cast<char *>(c->v);
    p.k_scale = c->k_scale;
    p.v_scale = c->v_scale;
    p.offsets = c->offsets;
    p.lens = c->lens;
    p.rows = c->total_rows;
    p.scale_blocks = c->scale_blocks;
    p.first_region = c->first_region;
    p.n_regions = (int)n_cells(s);
    p.heads = row_heads_of(s);
    return p;
}

}  // namespace

int launch_quantize(const aircache_shape_t *s, const aircache_ragged_t *c, aircache_quantized_t *out, cudaStream_t st) {
    QuantizeParams p = params_of(s, out);
    p.k = static_cast<const char *>(c->k);
    p.v = static_cast<const char *>(c->v);
    if (c->total_rows < p.rows) p.rows = c->total_rows;
    const int64_t blocks = (p.rows / kScaleRows + p.n_regions) * 2 * p.heads;   // below 2^31 / 64 * 16 + 1792 * 16
    const dim3 grid((unsigned)blocks);
    return s->head_dim == 64 ? launch_dependent(quantize_kernel<64>, grid, dim3(128), 0, st, p)
                             : launch_dependent(quantize_kernel<128>, grid, dim3(128), 0, st, p);
}

int launch_append_quantized(const aircache_shape_t *s, aircache_quantized_t *c, const void *k_new, const void *v_new,
                            cudaStream_t st) {
    QuantizeParams p = params_of(s, c);
    const dim3 grid((unsigned)p.n_regions), block(64 * p.heads);
    const char *k = static_cast<const char *>(k_new), *v = static_cast<const char *>(v_new);
    return s->head_dim == 64 ? launch_dependent(append_quantized_kernel<64>, grid, block, 0, st, p, c->lens, k, v)
                             : launch_dependent(append_quantized_kernel<128>, grid, block, 0, st, p, c->lens, k, v);
}

}  // namespace aircache
