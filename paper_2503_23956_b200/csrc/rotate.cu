// aircache_rotate: norms of queries and keys for each head, rotary positions and the store into the cache, one pass.
//
// For a head x (of a token at position pos):  y = x * rsqrt(mean(x^2) + eps) * w,  then every pair (a, b) of frequency i
// turns by pos * f_i:  (y_a c - y_b s, y_b c + y_a s).  2 bytes in and 2 bytes out per channel and some 10 operations: bound
// by memory.  A lane holds 8 channels (16 bytes), a head is 16 (8) lanes, so a warp takes two (four) heads of a token
// at a time, kBatch such loads under way at once; the pair of channels i and i + R/2 is a shuffle apart.  Heads of one token
// go to one warp where there are many tokens: cosines and sines, eight per lane, are then taken once for all of
// them.  Where there are few, they go to more warps.
//
// Angles: pos * f_i in fp32 is off by up to 2^-24 * pos radians, 0.03 at half a million.  The product is exact in fp64
// (31 + 24 bits), taken in turns and reduced to [-1/2, 1/2] there; sincospif does the rest.
#include "common.cuh"
#include "ptx.cuh"

namespace aircache {

namespace {

constexpr int kBatch = 4;

struct RotateParams {
    const char *q, *k, *v;
    char *q_out, *k_out, *v_out;
    int64_t q_l, q_t, q_h, k_l, k_t, k_h, v_l, v_t, v_h;          // strides in bytes
    int64_t qo_l, qo_t, qo_h, ko_l, ko_t, ko_h, vo_l, vo_t, vo_h;
    const int32_t *positions;
    const float *inv_freq;
    const uint16_t *q_weight, *k_weight;
    const int64_t *rows;
    int64_t n_rows, items;
    int n_tokens, Hq, Hkv, slots, parts, slots_per_part;
    int half, sec0, sec01;   // R / 2; frequencies of the first axis, of the first two
    float eps, factor;
};

__device__ __forceinline__ float2 bf16x2_f32(uint32_t w) { return make_float2(bf16lo(w), bf16hi(w)); }
__device__ __forceinline__ uint32_t f32_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(128) rotate_kernel(RotateParams p) {
    constexpr int LPH = D / 8;         // lanes of a head
    constexpr int HPW = 32 / LPH;      // heads a warp takes at a time
    const int lane = threadIdx.x & 31, l = lane % LPH, sub = lane / LPH;
    const int c0 = 8 * l;
    const bool turns = c0 < 2 * p.half;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5); item < p.items; item += (int64_t)gridDim.x * 4) {
        const int part = (int)(item % p.parts);
        const int64_t lt = item / p.parts;
        const int t = (int)(lt % p.n_tokens);
        const int64_t layer = lt / p.n_tokens;
        int64_t row = p.rows ? p.rows[t] : t;
        const bool stored = row >= 0 && row < p.n_rows;
        float c[8], s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (INTERLEAVED && (e & 1)) { c[e] = c[e - 1]; s[e] = s[e - 1]; continue; }
            c[e] = 1.f;
            s[e] = 0.f;
            if (turns) {
                const int i = INTERLEAVED ? (c0 + e) / 2 : (c0 < p.half ? c0 : c0 - p.half) + e;
                const int axis = i < p.sec0 ? 0 : (i < p.sec01 ? 1 : 2);
                const double angle = (double)p.positions[(int64_t)axis * p.n_tokens + t] * (double)p.inv_freq[i];
                const double turn = angle * 0.15915494309189535;   // 1 / (2 pi)
                sincospif(2.f * (float)(turn - rint(turn)), &s[e], &c[e]);
                c[e] *= p.factor;
                s[e] *= p.factor;
                if (!INTERLEAVED && c0 < p.half) s[e] = -s[e];   // of the first channel of a pair
            }
        }
        uint4 wq = make_uint4(0, 0, 0, 0), wk = wq;
        if (p.q_weight) wq = *reinterpret_cast<const uint4 *>(p.q_weight + layer * D + c0);
        if (p.k_weight) wk = *reinterpret_cast<const uint4 *>(p.k_weight + layer * D + c0);
        int partner = lane;
        if (!INTERLEAVED && turns) partner = lane + (c0 < p.half ? p.half / 8 : -(p.half / 8));

        const int first = part * p.slots_per_part;
        const int last = min(p.slots, first + p.slots_per_part);
        for (int base = first; base < last; base += HPW * kBatch) {
            uint4 x[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int h = base + b * HPW + sub;
                x[b] = make_uint4(0, 0, 0, 0);
                if (h < last) {
                    const char *src = h < p.Hq ? p.q + layer * p.q_l + t * p.q_t + h * p.q_h
                                    : h < p.Hq + p.Hkv ? p.k + layer * p.k_l + t * p.k_t + (h - p.Hq) * p.k_h
                                                       : p.v + layer * p.v_l + t * p.v_t + (h - p.Hq - p.Hkv) * p.v_h;
                    x[b] = *reinterpret_cast<const uint4 *>(src + 2 * c0);
                }
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (base + b * HPW >= last) break;   // (of the whole warp)
                const int h = base + b * HPW + sub;
                const bool is_v = h >= p.Hq + p.Hkv;
                float y[8];
                const uint32_t xw[4] = {x[b].x, x[b].y, x[b].z, x[b].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = bf16x2_f32(xw[i]);
                    y[2 * i] = f.x;
                    y[2 * i + 1] = f.y;
                }
                const uint16_t *weight = h < p.Hq ? p.q_weight : p.k_weight;
                if (p.q_weight || p.k_weight) {
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = fmaf(y[i], y[i], sum);
#pragma unroll
                    for (int o = 1; o < LPH; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    if (weight && !is_v) {
                        const float r = rsqrtf(sum * (1.f / D) + p.eps);
                        const uint4 w = h < p.Hq ? wq : wk;
                        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 f = bf16x2_f32(ww[i]);
                            y[2 * i] *= r * f.x;
                            y[2 * i + 1] *= r * f.y;
                        }
                    }
                }
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    if (INTERLEAVED) {
                        o[i] = y[i] * c[i] - y[i + 1] * s[i];
                        o[i + 1] = y[i + 1] * c[i] + y[i] * s[i];
                    } else {
                        o[i] = y[i] * c[i] + __shfl_sync(0xffffffffu, y[i], partner) * s[i];
                        o[i + 1] = y[i + 1] * c[i + 1] + __shfl_sync(0xffffffffu, y[i + 1], partner) * s[i + 1];
                    }
                }
                uint4 out;
                // (channels that do not turn keep their bits where there is no norm: 1 * y + y * 0 would make NaN of an infinity)
                const float *z = turns ? o : y;
                out.x = f32_bf16x2(z[0], z[1]);
                out.y = f32_bf16x2(z[2], z[3]);
                out.z = f32_bf16x2(z[4], z[5]);
                out.w = f32_bf16x2(z[6], z[7]);
                if (is_v) out = x[b];
                if (h < last && (h < p.Hq || stored)) {
                    char *dst = h < p.Hq ? p.q_out + layer * p.qo_l + t * p.qo_t + h * p.qo_h
                              : !is_v ? p.k_out + layer * p.ko_l + row * p.ko_t + (h - p.Hq) * p.ko_h
                                      : p.v_out + layer * p.vo_l + row * p.vo_t + (h - p.Hq - p.Hkv) * p.vo_h;
                    *reinterpret_cast<uint4 *>(dst + 2 * c0) = out;
                }
            }
        }
    }
}

}  // namespace

int launch_rotate(const aircache_rotary_t *r, const aircache_tokens_t *q, const aircache_tokens_t *k,
                  const aircache_tokens_t *v, const int32_t *positions, const float *inv_freq, const void *q_weight,
                  const void *k_weight, const aircache_tokens_t *q_out, const aircache_tokens_t *k_out,
                  const aircache_tokens_t *v_out, const int64_t *rows, int64_t n_rows, cudaStream_t st) {
    RotateParams p = {};
    auto side = [](const aircache_tokens_t *t, auto &data, int64_t &l, int64_t &tok, int64_t &h) {
        if (!t) return;
        data = static_cast<char *>(t->data);
        l = 2 * t->stride_layer;
        tok = 2 * t->stride_token;
        h = 2 * t->stride_head;
    };
    if (r->n_q_heads > 0) {
        side(q, p.q, p.q_l, p.q_t, p.q_h);
        side(q_out, p.q_out, p.qo_l, p.qo_t, p.qo_h);
    }
    if (r->n_kv_heads > 0) {
        side(k, p.k, p.k_l, p.k_t, p.k_h);
        side(k_out, p.k_out, p.ko_l, p.ko_t, p.ko_h);
        if (v) {
            side(v, p.v, p.v_l, p.v_t, p.v_h);
            side(v_out, p.v_out, p.vo_l, p.vo_t, p.vo_h);
        }
    }
    p.positions = positions;
    p.inv_freq = inv_freq;
    p.q_weight = (const uint16_t *)q_weight;
    p.k_weight = (const uint16_t *)k_weight;
    p.rows = rows;
    p.n_rows = n_rows;
    p.n_tokens = r->n_tokens;
    p.Hq = r->n_q_heads;
    p.Hkv = r->n_kv_heads;
    p.slots = p.Hq + p.Hkv + (v ? p.Hkv : 0);
    p.half = r->rotary_dim / 2;
    p.sec0 = r->sections[0];
    p.sec01 = r->sections[0] + r->sections[1];
    p.eps = r->eps;
    p.factor = r->factor;
    int dev = 0, sms = 0, rc = current_device(&dev, &sms);
    if (rc) return rc;
    // A warp takes all heads of a token from half the warps that the GPU holds on; below, kBatch loads of them.
    const int64_t tokens = (int64_t)r->n_layers * r->n_tokens;
    const int step = 32 / (r->head_dim / 8) * kBatch;
    p.slots_per_part = tokens >= (int64_t)sms * 32 ? p.slots : step;
    p.parts = (p.slots + p.slots_per_part - 1) / p.slots_per_part;
    p.items = tokens * p.parts;
    const int64_t blocks = (p.items + 3) / 4;
    const dim3 grid((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30)));
    if (r->head_dim == 64)
        return r->interleaved ? launch_dependent(rotate_kernel<64, true>, grid, dim3(128), 0, st, p)
                              : launch_dependent(rotate_kernel<64, false>, grid, dim3(128), 0, st, p);
    return r->interleaved ? launch_dependent(rotate_kernel<128, true>, grid, dim3(128), 0, st, p)
                          : launch_dependent(rotate_kernel<128, false>, grid, dim3(128), 0, st, p);
}

}  // namespace aircache
