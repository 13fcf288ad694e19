// aircache_rotate: norms of queries and keys for each head, rotary positions and the store into the cache, one pass.
//
// For a head x (of a token at position pos):  y = x * rsqrt(mean(x^2) + eps) * w,  then every pair (a, b) of frequency i
// turns by pos * f_i:  (y_a c - y_b s, y_b c + y_a s).  2 bytes in and 2 bytes out per channel: bound by memory, once the
// arithmetic is kept small.  A head is 16 (8) lanes, so a warp takes two (four) heads of a token at a time, kBatch such loads
// under way at once.  A lane holds both channels of its four pairs (8 bytes from either half of the rotated channels, or 16
// consecutive bytes in the interleaved layout): no exchange between lanes but for the norm's sum, and four cosines and
// sines a token.  (With 16 consecutive bytes per lane in both layouts, partners fetched by shuffles: 174 us for 27136
// tokens of 28 + 2 * 4 heads.)  Heads of one token go to one warp where there are many tokens: the angles are
// then taken once for all of them.  Where there are few, they go to more warps.  27136 tokens, us: 117 with four loads under
// way and 20 warps an SM, 103 with two and 32 (4.8 TB/s; the norm's sum takes 13 of it, the angles 4; 64 registers a thread, 3 to 8 of them spilled).  Measured and not kept: the next
// loads asked for ahead of the angles and of a batch's arithmetic (107), two numbers an instruction (105 to 109), the
// sums of a batch side by side (109), one load under way and 40 warps (118).
//
// Angles: pos * f_i in fp32 is off by up to 2^-24 * pos radians, 0.03 at half a million.  The product is exact in fp64
// (31 + 24 bits), taken in turns and reduced to [-1/2, 1/2] there; sincospif does the rest.
#include "common.cuh"
#include "ptx.cuh"

namespace aircache {

namespace {

constexpr int kBatch = 2;

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

template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(128, 8) rotate_kernel(RotateParams p) {
    constexpr int LPH = D / 8;         // lanes of a head
    constexpr int HPW = 32 / LPH;      // heads a warp takes at a time
    const int lane = threadIdx.x & 31, l = lane % LPH, sub = lane / LPH;
    // the lane's channels: lo .. lo + 3 and hi .. hi + 3, channel lo + e turns with hi + e (interleaved: with its neighbour)
    const bool turns = 4 * l < p.half;
    const int lo = turns && !INTERLEAVED ? 4 * l : 8 * l, hi = turns && !INTERLEAVED ? p.half + 4 * l : lo + 4;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5); item < p.items; item += (int64_t)gridDim.x * 4) {
        const int part = (int)(item % p.parts);
        const int64_t lt = item / p.parts;
        const int t = (int)(lt % p.n_tokens);
        const int64_t layer = lt / p.n_tokens;
        const int64_t row = p.rows ? p.rows[t] : t;
        const bool stored = row >= 0 && row < p.n_rows;
        const int first = part * p.slots_per_part, last = min(p.slots, first + p.slots_per_part);
        float c[4], s[4];   // of pairs 4 l .. 4 l + 3
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = 1.f;
            s[e] = 0.f;
            if (turns) {
                const int i = 4 * l + e;
                const int axis = i < p.sec0 ? 0 : (i < p.sec01 ? 1 : 2);
                const double angle = (double)p.positions[(int64_t)axis * p.n_tokens + t] * (double)p.inv_freq[i];
                const double turn = angle * 0.15915494309189535;   // 1 / (2 pi)
                sincospif(2.f * (float)(turn - rint(turn)), &s[e], &c[e]);
                c[e] *= p.factor;
                s[e] *= p.factor;
            }
        }
        // heads [from, to) of the queries or keys
        auto rotate_heads = [&](const char *src, int64_t src_head, char *dst, int64_t dst_head, const uint16_t *weight, int from, int to) {
            float w[8];
            if (weight) {
                const uint2 a = *reinterpret_cast<const uint2 *>(weight + layer * D + lo), b = *reinterpret_cast<const uint2 *>(weight + layer * D + hi);
                w[0] = bf16lo(a.x); w[1] = bf16hi(a.x); w[2] = bf16lo(a.y); w[3] = bf16hi(a.y);
                w[4] = bf16lo(b.x); w[5] = bf16hi(b.x); w[6] = bf16lo(b.y); w[7] = bf16hi(b.y);
            }
            src += (from + sub) * src_head;
            dst += (from + sub) * dst_head;
            const int64_t src_step = HPW * src_head, dst_step = HPW * dst_head;
            for (int base = from; base < to; base += HPW * kBatch) {
                uint2 x[kBatch][2];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    x[b][0] = x[b][1] = make_uint2(0, 0);
                    if (base + b * HPW + sub < to) {
                        x[b][0] = *reinterpret_cast<const uint2 *>(src + 2 * lo);
                        x[b][1] = *reinterpret_cast<const uint2 *>(src + 2 * hi);
                    }
                    src += src_step;
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    if (base + b * HPW >= to) break;   // (of the whole warp)
                    float y[8] = {bf16lo(x[b][0].x), bf16hi(x[b][0].x), bf16lo(x[b][0].y), bf16hi(x[b][0].y),
                                  bf16lo(x[b][1].x), bf16hi(x[b][1].x), bf16lo(x[b][1].y), bf16hi(x[b][1].y)};
                    if (weight) {
                        float sum = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum = fmaf(y[e], y[e], sum);
#pragma unroll
                        for (int o = 1; o < LPH; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                        const float r = rsqrtf(sum * (1.f / D) + p.eps);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] *= r * w[e];
                    }
                    if (turns) {   // (channels that do not turn keep their value: 1 * y + 0 * y would make NaN of an infinity)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float &a = y[INTERLEAVED ? 2 * e : e], &b2 = y[INTERLEAVED ? 2 * e + 1 : 4 + e];
                            const float turned = a * c[e] - b2 * s[e];
                            b2 = b2 * c[e] + a * s[e];
                            a = turned;
                        }
                    }
                    if (base + b * HPW + sub < to) {
                        *reinterpret_cast<uint2 *>(dst + 2 * lo) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
                        *reinterpret_cast<uint2 *>(dst + 2 * hi) = make_uint2(pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                    }
                    dst += dst_step;
                }
            }
        };
        if (first < p.Hq)
            rotate_heads(p.q + layer * p.q_l + t * p.q_t, p.q_h, p.q_out + layer * p.qo_l + t * p.qo_t, p.qo_h, p.q_weight, first,
                         min(last, p.Hq));
        if (last > p.Hq && stored) {
            if (first < p.Hq + p.Hkv)
                rotate_heads(p.k + layer * p.k_l + t * p.k_t, p.k_h, p.k_out + layer * p.ko_l + row * p.ko_t, p.ko_h, p.k_weight,
                             max(first - p.Hq, 0), min(last - p.Hq, p.Hkv));
            for (int h = max(first - p.Hq - p.Hkv, 0) + sub; h < last - p.Hq - p.Hkv; h += HPW)
                *reinterpret_cast<uint4 *>(p.v_out + layer * p.vo_l + row * p.vo_t + h * p.vo_h + 16 * l) =
                    *reinterpret_cast<const uint4 *>(p.v + layer * p.v_l + t * p.v_t + h * p.v_h + 16 * l);
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
