// aircache_decode_attn_quantized: single-token attention over the ragged cache of 8 bits, all regions in one launch.
//
//   out_h = sum_j p_j v_j / sum_j p_j,  p_j = exp2(scale log2(e) <q_h, k_j> - ref),  k_j, v_j = codes * their block's scale
//
// Bound by memory: an element is one byte and is read once; the two products do 4 G flop for it (G = 7 or 8 query
// heads share a KV head), far too much for FMAs beside the conversions, so both run on mma.sync m16n8k16 in fp16, which holds
// every e4m3 number exactly.  As in decode.cu they are taken transposed, S^T = K Q^T and O^T = V^T P^T: 16 keys
// (channels) are the rows and the query heads the 8 columns of a tile.
//
// Work.  A tile is 16 rows of a region (one KV head's worth of them per warp; a block of scales is four tiles).  The tiles
// of all items (an item is a region; or a region and KV head, where these do not outnumber the SMs) form one list, CTA c takes an
// equal contiguous share of it.  In a CTA, warp (head, sub) takes every SUBS-th tile of the share.  What a warp reads it reads for
// itself: every lane copies the very bytes that it will need for its fragments into its own places of a ring in shared
// memory (cp.async, 16 bytes), so there is no barrier and no bank conflict, and no ldmatrix that would need 16-bit elements:
//   K fragments   lane (g, t) = (lane / 4, lane % 4) holds channels 16t..16t+15 (and 64+16t..) of keys g and g + 8.  Which
//                 channels form a step of the product is free as long as q is laid out alike.
//   V fragments   lane (g, t) holds channels 16g..16g+15 of keys 2t, 2t+1, 2t+8, 2t+9, the keys whose weights movmatrix
//                 brings it; a byte permutation pairs two keys.
// A ring slot is refilled when its tile is done; the ring runs on over the end of an item.  At the end of an item's part the SUBS states of
// a head merge in a tree; an item that lies in one CTA is written, otherwise the CTA stores an unnormalised partial
// and takes a ticket of the item, and the one that draws the last merges all of them in order.  Nobody waits.
//
// Numbers.  q is scaled by a power of two per head, so that its largest magnitude is 2^7 to 2^8 in fp16: what is 2^-32 of it is lost.
// The reference of the softmax follows the largest logit lazily (it moves when one is more than 2^4 above), p <= 2^4.  p
// times its block's V scale over the largest V scale seen, times 2^11, is split into an fp16 head and remainder (22 bits).  Sums in fp32.
#include <atomic>

#include "common.cuh"
#include "ptx.cuh"
#include "quantize.cuh"

namespace aircache {

namespace {

struct DecodeQParams {
    const char *k, *v;
    const float *k_scale, *v_scale;
    const int64_t *offsets;
    const int32_t *lens;
    const uint16_t *q;   // [items, heads of an item, D]
    float *out;          // the same
    int32_t *tickets;    // [items], zero between calls
    float *partials;     // [2 * CTAs][slot]
    int64_t rows, scale_blocks, first_region;
    int items, split;    // split: KV heads per region where an item is a (region, head), else 1
    int row_heads;       // KV heads of a row in memory
    int Hq, G;           // query heads of an item, of a KV head
    float sl2;           // scale * log2(e)
};

constexpr int kTile = 16;
constexpr float kLift = 2048.f;   // of the weights, above fp16's subnormal numbers

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void *src, bool valid) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(valid ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 f16x2_f32(uint32_t h) {
    float2 r;
    asm("{\n.reg .f16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}\n" : "=f"(r.x), "=f"(r.y) : "r"(h));
    return r;
}

template <int D, int HEADS, int NT>
struct DecodeQCfg {
    static constexpr int WARPS = NT == 2 ? 8 : 16;
    static constexpr int SUBS = WARPS / HEADS;
    static constexpr int THREADS = WARPS * 32;
    static constexpr int CHUNKS = D / 64;                  // 64 channels of K: 16 per lane
    static constexpr int MT = D / 16;                      // channel tiles of O^T
    static constexpr int STAGE = 2 * kTile * D;            // bytes of a warp's tile, K and V
    static constexpr int STAGES = NT == 2 ? (D == 128 ? 4 : 8) : (D == 128 ? 2 : 4);
    static constexpr int STATE = NT * (MT * 4 + 4);        // floats of a lane's state
    static constexpr int MERGE = HEADS * (SUBS / 2) * STATE * 32 * 4;
    static constexpr int RING = WARPS * STAGES * STAGE;
    static constexpr int SCALES = WARPS * STAGES * 8;
    static constexpr int TABLES = (3 * kMaxRegions + 1) * 4;
    static constexpr int SMEM = RING + SCALES + MERGE + TABLES;
    static_assert(SMEM <= 232448 - 1024, "shared memory of a block");
};

// largest i with P[i] <= u (P non-decreasing, P[0] = 0, u < P[n])
__device__ __forceinline__ int find_item(const int *P, int n, int u) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (P[mid] <= u) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <int D, int HEADS, int NT>
__global__ void __launch_bounds__(DecodeQCfg<D, HEADS, NT>::THREADS, 1) decode_quantized_kernel(DecodeQParams p) {
    using C = DecodeQCfg<D, HEADS, NT>;
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char *s_ring = smem;
    float *s_scales = reinterpret_cast<float *>(smem + C::RING);
    float *s_merge = reinterpret_cast<float *>(smem + C::RING + C::SCALES);
    int *s_P = reinterpret_cast<int *>(smem + C::RING + C::SCALES + C::MERGE);   // [items + 1] first tile of an item
    int *s_off = s_P + kMaxRegions + 1, *s_len = s_off + kMaxRegions;
    __shared__ int s_sum[C::WARPS];
    __shared__ int s_last;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int head = warp % HEADS, sub = warp / HEADS;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // first tile, first row and rows of every item
    {
        constexpr int PER = (kMaxRegions + C::THREADS - 1) / C::THREADS;
        int n[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int item = tid * PER + i;
            n[i] = 0;
            if (item < p.items) {
                const int r = item / p.split;
                const int len = rows_in_use(p.offsets, p.lens, r, p.rows, p.first_region, p.scale_blocks);
                s_off[item] = (int)p.offsets[r];
                s_len[item] = len;
                n[i] = (len + kTile - 1) / kTile;
            }
            sum += n[i];
        }
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) s_sum[warp] = incl;
        __syncthreads();
        int before = incl - sum;
        for (int w = 0; w < warp; ++w) before += s_sum[w];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int item = tid * PER + i;
            if (item <= p.items) s_P[item] = before;
            before += n[i];
        }
        __syncthreads();
    }
    const int total = s_P[p.items], cta = blockIdx.x;
    for (int i = cta; i < p.items; i += gridDim.x)
        if (s_len[i] == 0)
            for (int e = tid; e < p.Hq * D; e += C::THREADS) p.out[(int64_t)i * p.Hq * D + e] = 0.f;
    const int ctas = min((int)gridDim.x, total);   // each of them has a tile
    if (cta >= ctas) return;
    const int t0 = (int)((int64_t)total * cta / ctas), t1 = (int)((int64_t)total * (cta + 1) / ctas);

    const uint32_t ring = smem_u32(s_ring) + warp * (C::STAGES * C::STAGE) + lane * 16;
    const uint32_t scales = smem_u32(s_scales) + warp * (C::STAGES * 8);
    const float *my_scales = s_scales + warp * (C::STAGES * 2);
    const unsigned char *my_ring = s_ring + warp * (C::STAGES * C::STAGE) + lane * 16;
    const int64_t pitch = (int64_t)p.row_heads * D;

    // the warp's tiles: tau = sub mod SUBS in [t0, t1)
    const int first_item = find_item(s_P, p.items, t0);
    int ask = t0 + (sub - t0 % C::SUBS + C::SUBS) % C::SUBS, ask_item = first_item, ask_stage = 0;
    auto issue = [&]() {   // the next tile into the next stage of the ring
        if (ask < t1) {
            while (ask >= s_P[ask_item + 1]) ++ask_item;
            const int row0 = (ask - s_P[ask_item]) * kTile, n = s_len[ask_item];
            const int64_t o = s_off[ask_item];
            const int r = ask_item / p.split;
            const int h = p.split > 1 ? ask_item - r * p.split : head;
            const int64_t base = (o + row0) * pitch + h * D;
            const uint32_t dst = ring + ask_stage * C::STAGE;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int key = g + 8 * i;
                const bool valid = row0 + key < n;
                const char *src = p.k + base + (valid ? key * pitch : 0) + t * 16;
#pragma unroll
                for (int c = 0; c < C::CHUNKS; ++c) cp_async16(dst + (i * C::CHUNKS + c) * 512, src + c * 64, valid);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = 2 * t + (i & 1) + 8 * (i >> 1);
                const bool valid = row0 + key < n;
                const char *src = p.v + base + (valid ? key * pitch : 0) + g * (D / 8);
                if (D == 128) cp_async16(dst + kTile * D + i * 512, src, valid);
                else cp_async8(dst + kTile * D + i * 256 - lane * 8, src, valid);
            }
            if (lane < 2) {
                const int64_t at = (o / kScaleRows + p.first_region + r + row0 / kScaleRows) * p.row_heads + h;
                cp_async4(scales + ask_stage * 8 + lane * 4, (lane ? p.v_scale : p.k_scale) + at);
            }
            ask += C::SUBS;
        }
        cp_commit();
        ask_stage = ask_stage + 1 == C::STAGES ? 0 : ask_stage + 1;
    };
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) issue();

    int tau = t0 + (sub - t0 % C::SUBS + C::SUBS) % C::SUBS, stage = 0;
    for (int item = first_item; item < p.items && s_P[item] < t1; ++item) {
        const int item_first = s_P[item], item_end = s_P[item + 1];
        if (item_first == item_end) continue;
        const int n = s_len[item], end = min(t1, item_end);

        // the item's queries as fp16 fragments: columns are the heads of the KV group, lane (g, t) holds head g (+ 8)
        uint32_t qf[NT][C::CHUNKS][8];
        float f[NT][2];   // logits of heads 2t, 2t + 1 (+ 8) from the products, without the K scale
        const uint16_t *q_item = p.q + ((int64_t)item * p.Hq + head * p.G) * D;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int h = nt * 8 + g;
            uint4 x[C::CHUNKS][2];
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[c][i] = make_uint4(0, 0, 0, 0);
                    if (h < p.G) x[c][i] = *reinterpret_cast<const uint4 *>(q_item + h * D + c * 64 + t * 16 + i * 8);
                    const uint32_t w[4] = {x[c][i].x, x[c][i].y, x[c][i].z, x[c][i].w};
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const uint32_t l = w[a] & 0x7fffu, u = w[a] >> 16 & 0x7fffu;
                        top = max(top, max(l < 0x7f80 ? l : 0, u < 0x7f80 ? u : 0));
                    }
                }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // 2^e brings the largest magnitude to [2^7, 2^8); both 2^e and 2^-e are normal numbers
            const int e = min(max(134 - (int)(top >> 7), -119), 126);
            const float up = __uint_as_float((uint32_t)(127 + e) << 23), down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t w[4] = {x[c][i].x, x[c][i].y, x[c][i].z, x[c][i].w};
#pragma unroll
                    for (int a = 0; a < 4; ++a) qf[nt][c][i * 4 + a] = f16x2(bf16lo(w[a]) * up, bf16hi(w[a]) * up);
                }
            f[nt][0] = __shfl_sync(0xffffffffu, down, 8 * t) * p.sl2;
            f[nt][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4) * p.sl2;
        }
        if (item + 1 < p.items && item_end < t1) {   // the next item's queries on their way
            const char *next = reinterpret_cast<const char *>(p.q + (int64_t)(item + 1) * p.Hq * D);
            for (int i = tid; i * 128 < p.Hq * D * 2; i += C::THREADS) prefetch_l2(next + i * 128);
        }

        float acc[NT][C::MT][4], ref[NT][2], sum[NT][2], v_top = 0.f, v_inv = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < C::MT; ++c) acc[nt][c][0] = acc[nt][c][1] = acc[nt][c][2] = acc[nt][c][3] = 0.f;
            ref[nt][0] = ref[nt][1] = -INFINITY;
            sum[nt][0] = sum[nt][1] = 0.f;
        }

        for (; tau < end; tau += C::SUBS) {
            cp_wait<C::STAGES - 2>();
            __syncwarp();
            issue();
            const unsigned char *tile = my_ring + stage * C::STAGE;
            const float ks = my_scales[stage * 2], vs = my_scales[stage * 2 + 1];
            stage = stage + 1 == C::STAGES ? 0 : stage + 1;

            float s[NT][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[nt][0][i] = s[nt][1][i] = 0.f;
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c) {
                const uint4 ka = *reinterpret_cast<const uint4 *>(tile + c * 512);
                const uint4 kb = *reinterpret_cast<const uint4 *>(tile + (C::CHUNKS + c) * 512);
                const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t a0 = e4m3x2_f16x2(wa[w] & 0xffffu), a2 = e4m3x2_f16x2(wa[w] >> 16);
                    const uint32_t a1 = e4m3x2_f16x2(wb[w] & 0xffffu), a3 = e4m3x2_f16x2(wb[w] >> 16);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16_16816(s[nt][w & 1], a0, a1, a2, a3, qf[nt][c][2 * w], qf[nt][c][2 * w + 1]);
                }
            }
            const int rows = n - (tau - item_first) * kTile;   // of the tile, 16 or more unless it is the item's last
            bool moves = false;
            float x[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[nt][i] = (s[nt][0][i] + s[nt][1][i]) * (f[nt][i & 1] * ks);
                if (rows < kTile) {
                    if (g >= rows) x[nt][0] = x[nt][1] = -INFINITY;
                    if (g + 8 >= rows) x[nt][2] = x[nt][3] = -INFINITY;
                }
                moves = moves || fmaxf(x[nt][0], x[nt][2]) > ref[nt][0] + 4.f || fmaxf(x[nt][1], x[nt][3]) > ref[nt][1] + 4.f;
            }
            if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float top = fmaxf(x[nt][j], x[nt][j + 2]);
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                        const float now = fmaxf(fmaxf(ref[nt][j], top), -1e30f);
                        const float shrink = fast_exp2(ref[nt][j] - now);
                        ref[nt][j] = now;
                        sum[nt][j] *= shrink;
#pragma unroll
                        for (int c = 0; c < C::MT; ++c) {
                            acc[nt][c][j] *= shrink;
                            acc[nt][c][j + 2] *= shrink;
                        }
                    }
            }
            if (vs > v_top) {   // (all lanes alike)
                const float shrink = v_top / vs;
                v_top = vs;
                v_inv = kLift / vs;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < C::MT; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[nt][c][i] *= shrink;
            }
            const float vf = vs * v_inv;
            uint32_t head_b[NT][2], rest_b[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {   // keys g (i = 0) and g + 8
                    const float p0 = fast_exp2(x[nt][2 * i] - ref[nt][0]), p1 = fast_exp2(x[nt][2 * i + 1] - ref[nt][1]);
                    sum[nt][0] += p0;
                    sum[nt][1] += p1;
                    const uint32_t hi = f16x2(p0 * vf, p1 * vf);
                    const float2 back = f16x2_f32(hi);
                    head_b[nt][i] = movmatrix_trans(hi);
                    rest_b[nt][i] = movmatrix_trans(f16x2(fmaf(p0, vf, -back.x), fmaf(p1, vf, -back.y)));
                }
            uint32_t vw[4][C::MT / 2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (D == 128) {
                    const uint4 x4 = *reinterpret_cast<const uint4 *>(tile + kTile * D + i * 512);
                    vw[i][0] = x4.x; vw[i][1] = x4.y; vw[i][C::MT / 2 - 2] = x4.z; vw[i][C::MT / 2 - 1] = x4.w;
                } else {
                    const uint2 x2 = *reinterpret_cast<const uint2 *>(tile + kTile * D + i * 256 - lane * 8);
                    vw[i][0] = x2.x; vw[i][1] = x2.y;
                }
            }
#pragma unroll
            for (int w = 0; w < C::MT / 2; ++w) {
                // channels 4w..4w+3 of this lane's stretch, two keys abreast
                const uint32_t l01 = __byte_perm(vw[0][w], vw[1][w], 0x5140), u01 = __byte_perm(vw[0][w], vw[1][w], 0x7362);
                const uint32_t l23 = __byte_perm(vw[2][w], vw[3][w], 0x5140), u23 = __byte_perm(vw[2][w], vw[3][w], 0x7362);
                const uint32_t a0 = e4m3x2_f16x2(l01 & 0xffffu), a1 = e4m3x2_f16x2(l01 >> 16);
                const uint32_t a2 = e4m3x2_f16x2(l23 & 0xffffu), a3 = e4m3x2_f16x2(l23 >> 16);
                const uint32_t b0 = e4m3x2_f16x2(u01 & 0xffffu), b1 = e4m3x2_f16x2(u01 >> 16);
                const uint32_t b2 = e4m3x2_f16x2(u23 & 0xffffu), b3 = e4m3x2_f16x2(u23 >> 16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_f16_16816(acc[nt][2 * w], a0, a1, a2, a3, head_b[nt][0], head_b[nt][1]);
                    mma_f16_16816(acc[nt][2 * w + 1], b0, b1, b2, b3, head_b[nt][0], head_b[nt][1]);
                    mma_f16_16816(acc[nt][2 * w], a0, a1, a2, a3, rest_b[nt][0], rest_b[nt][1]);
                    mma_f16_16816(acc[nt][2 * w + 1], b0, b1, b2, b3, rest_b[nt][0], rest_b[nt][1]);
                }
            }
        }

        // the end of the item's part: sums over the lanes of a head, true units, then the tree over the head's warps
        const float unit = v_top * (1.f / kLift);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], 4);
                sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], 8);
                sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], 16);
#pragma unroll
                for (int c = 0; c < C::MT; ++c) {
                    acc[nt][c][j] *= unit;
                    acc[nt][c][j + 2] *= unit;
                }
            }
#pragma unroll
        for (int half = C::SUBS / 2; half >= 1; half >>= 1) {
            if (sub >= half && sub < 2 * half) {
                float *to = s_merge + (head * (C::SUBS / 2) + sub - half) * (C::STATE * 32) + lane;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float *at = to + nt * (C::MT * 4 + 4) * 32;
                    at[0] = ref[nt][0]; at[32] = ref[nt][1]; at[64] = sum[nt][0]; at[96] = sum[nt][1];
#pragma unroll
                    for (int c = 0; c < C::MT; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) at[(4 + c * 4 + i) * 32] = acc[nt][c][i];
                }
            }
            __syncthreads();
            if (sub < half) {
                const float *from = s_merge + (head * (C::SUBS / 2) + sub) * (C::STATE * 32) + lane;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float *at = from + nt * (C::MT * 4 + 4) * 32;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float other = at[32 * j], now = fmaxf(fmaxf(ref[nt][j], other), -1e30f);
                        const float mine = fast_exp2(ref[nt][j] - now), theirs = fast_exp2(other - now);
                        ref[nt][j] = now;
                        sum[nt][j] = sum[nt][j] * mine + at[64 + 32 * j] * theirs;
#pragma unroll
                        for (int c = 0; c < C::MT; ++c) {
                            acc[nt][c][j] = acc[nt][c][j] * mine + at[(4 + c * 4 + j) * 32] * theirs;
                            acc[nt][c][j + 2] = acc[nt][c][j + 2] * mine + at[(4 + c * 4 + j + 2) * 32] * theirs;
                        }
                    }
                }
            }
            __syncthreads();
        }

        const bool whole = item_first >= t0 && item_end <= t1;
        const int64_t slot_floats = partial_slot_floats(p.Hq, D);
        float *slot = p.partials + (2 * (int64_t)cta + (item_first >= t0 ? 1 : 0)) * slot_floats;
        if (sub == 0) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int h = nt * 8 + 2 * t + j;
                    if (h >= p.G) continue;
                    const int hq = head * p.G + h;
                    const float times = whole ? (sum[nt][j] > 0.f || sum[nt][j] != sum[nt][j] ? 1.f / sum[nt][j] : 0.f) : 1.f;
                    float *to = (whole ? p.out + ((int64_t)item * p.Hq + hq) * D : slot + (int64_t)hq * D) + g * (D / 8);
#pragma unroll
                    for (int c = 0; c < C::MT; c += 2)
                        *reinterpret_cast<float4 *>(to + 2 * c) =
                            make_float4(acc[nt][c][j] * times, acc[nt][c][j + 2] * times, acc[nt][c + 1][j] * times,
                                        acc[nt][c + 1][j + 2] * times);
                    if (!whole && g == 0) {
                        slot[(int64_t)p.Hq * D + hq] = ref[nt][j];
                        slot[(int64_t)p.Hq * (D + 1) + hq] = sum[nt][j];
                    }
                }
        }
        if (!whole) {
            __syncthreads();
            // the CTAs that have a part of the item, in order: tile u belongs to CTA ((u + 1) * ctas - 1) / total
            const int c_first = (int)(((int64_t)(item_first + 1) * ctas - 1) / total);
            const int c_last = (int)(((int64_t)item_end * ctas - 1) / total);
            if (tid == 0) {
                __threadfence();
                s_last = atomicAdd(p.tickets + item, 1) == c_last - c_first;
                __threadfence();
            }
            __syncthreads();
            if (s_last) {
                for (int e = tid; e < p.Hq * D; e += C::THREADS) {
                    const int hq = e / D;
                    float m = -1e30f, o = 0.f, l = 0.f;
                    for (int c = c_first; c <= c_last; ++c) {
                        const float *from = p.partials + (2 * (int64_t)c + (c == c_first ? 1 : 0)) * slot_floats;
                        const float cm = __ldcg(from + (int64_t)p.Hq * D + hq), cl = __ldcg(from + (int64_t)p.Hq * (D + 1) + hq);
                        const float co = __ldcg(from + e);
                        const float now = fmaxf(m, cm), mine = fast_exp2(m - now), theirs = fast_exp2(cm - now);
                        m = now;
                        l = l * mine + cl * theirs;
                        o = o * mine + co * theirs;
                    }
                    p.out[(int64_t)item * p.Hq * D + e] = l > 0.f || l != l ? o / l : 0.f;
                }
                if (tid == 0) p.tickets[item] = 0;
            }
        }
    }
    cp_wait<0>();
}

template <int D, int HEADS, int NT>
int launch_t(const DecodeQParams &p, int ctas, int dev, cudaStream_t st) {
    using C = DecodeQCfg<D, HEADS, NT>;
    static std::atomic<uint64_t> allowed[kMaxDevices];
    const int rc = allow_shared_memory((const void *)decode_quantized_kernel<D, HEADS, NT>, C::SMEM, dev, allowed);
    if (rc) return rc;
    return launch_dependent(decode_quantized_kernel<D, HEADS, NT>, dim3(ctas), dim3(C::THREADS), C::SMEM, st, p);
}

template <int D, int HEADS>
int launch_g(const DecodeQParams &p, int ctas, int dev, cudaStream_t st) {
    return p.G > 8 ? launch_t<D, HEADS, 2>(p, ctas, dev, st) : launch_t<D, HEADS, 1>(p, ctas, dev, st);
}

template <int D>
int launch_d(const DecodeQParams &p, int heads, int ctas, int dev, cudaStream_t st) {
    switch (heads) {
        case 1: return launch_g<D, 1>(p, ctas, dev, st);
        case 2: return launch_g<D, 2>(p, ctas, dev, st);
        case 4: return launch_g<D, 4>(p, ctas, dev, st);
        case 8: return launch_g<D, 8>(p, ctas, dev, st);
        default: return AIRCACHE_ERR_UNSUPPORTED;
    }
}

}  // namespace

int launch_decode_quantized(const aircache_shape_t *s, const aircache_quantized_t *c, const void *q, float *out,
                            void *ws, cudaStream_t st) {
    const WsLayout w = ws_layout(s);
    int dev = 0, sms = 0, rc = current_device(&dev, &sms);
    if (rc) return rc;
    const int ctas = sms < kMaxDecodeCtas ? sms : kMaxDecodeCtas;
    DecodeQParams p = {};
    p.k = static_cast<const char *>(c->k);
    p.v = static_cast<const char *>(c->v);
    p.k_scale = c->k_scale;
    p.v_scale = c->v_scale;
    p.offsets = c->offsets;
    p.lens = c->lens;
    p.q = static_cast<const uint16_t *>(q);
    p.out = out;
    p.tickets = ws_ptr<int32_t>(ws, w.tickets);
    p.partials = ws_ptr<float>(ws, w.partials);
    p.rows = c->total_rows;
    p.scale_blocks = c->scale_blocks;
    p.first_region = c->first_region;
    p.row_heads = row_heads_of(s);
    p.G = s->n_q_heads / s->n_kv_heads;
    p.items = (int)n_cells(s);
    p.split = 1;
    p.sl2 = s->scale * kLog2e;
    int heads = p.row_heads;
    // So few regions that (region, KV head) pairs do not outnumber the SMs: an item is such a pair (decode.cu).
    if (heads > 1 && p.items * heads <= ctas) {
        p.split = heads;
        p.items *= heads;
        heads = 1;
    }
    p.Hq = heads * p.G;
    return s->head_dim == 64 ? launch_d<64>(p, heads, ctas, dev, st) : launch_d<128>(p, heads, ctas, dev, st);
}

}  // namespace aircache
