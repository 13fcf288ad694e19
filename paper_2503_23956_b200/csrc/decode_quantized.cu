// aircache_decode_attn_quantized: single-token attention over the ragged cache of 8 bits, all regions in one launch.
//
//   out_h = sum_j p_j v_j / sum_j p_j,  p_j = exp2(scale log2(e) <q_h, k_j> - ref),  k_j, v_j = codes * their block's scale
//
// Bound by memory: an element is one byte and is read once; the two products do 4 G flop for it (G = 7 or 8 query
// heads share a KV head), far too much for FMAs beside the conversions, so both run on mma.sync m16n8k16 in fp16, which holds
// every e4m3 number exactly.  As in decode.cu they are taken transposed, S^T = K Q^T and O^T = V^T P^T: 16 keys
// (channels) are the rows and the query heads the 8 columns of a tile.
//
// Work.  A tile is 32 rows of a region (one KV head's worth of them per warp; a block of scales is two tiles); an item is a
// region, or a region and KV head where these do not outnumber the SMs.
//   More items than SMs: the tiles of all items form one list, of which CTA c takes an equal contiguous share; a table of
//   the items is built in shared memory.
//   Else: an item is cut into pieces of equal size for as many CTAs, and stays whole where that costs less than the merge of
//   pieces would.  Every warp plans this in registers.
// In a CTA, warp (head, sub) takes every SUBS-th tile of the CTA's part, through a ring of its own in shared memory that
// one of its lanes fills by TMA (boxes of 16 rows of one head, 128-byte swizzle, mbarriers): no warp waits for another.  The fragments
// are read as 16 bytes per lane, since ldmatrix has no form for 8-bit elements of 16-bit products:
//   K fragments   lane (g, t) = (lane / 4, lane % 4) holds channels 32t..32t+31 of keys g and g + 8.  Which
//                 channels form a step of the product is free as long as q is laid out alike.
//   V fragments   lane (g, t) holds channels 16g..16g+15 of keys 2t, 2t+1, 2t+8, 2t+9, the keys whose weights movmatrix
//                 brings it; a byte permutation pairs two keys.
// A ring runs on over the end of an item.  There the SUBS states of a head merge through the ring stages just read;
// an item that lies in one CTA is written, otherwise the CTA stores an unnormalised partial
// and takes a ticket of the item, and the one that draws the last merges all of them in order.  Nobody waits.
//
// Numbers.  q is scaled by a power of two per head, so that its largest magnitude is 2^7 to 2^8 in fp16: what is 2^-32 of it is lost.
// The reference of the softmax follows the largest logit lazily (it moves when one is more than 2^4 above), p <= 2^4.  p
// times its block's V scale over the largest V scale seen (2^-116 at least), times 2^11, is split into an fp16 head and remainder (22 bits).  Sums in fp32.
//
// Measured (one B200, us a call; bytes at 6.54 TB/s in brackets): 64 sequences of 548 rows in 28 layers, 28 / 4 heads of 128: 189 [160], 207 to 214
// in a second of calls back to back under the power cap; 640 cells of one KV head 80 [61]; one image 11.9 [3.9], four videos 39.0 [20.4].  A tile takes a
// warp some 2270 cycles, the memory's rate leaves it 2700: conversions, 2 x 24 products and the softmax, 500 instructions.  16 warps of
// 16-row tiles: 221 us for the 184 that this took then; items of one head for many regions: 43 for 37.
#include <cuda.h>

#include <atomic>

#include "common.cuh"
#include "ptx.cuh"
#include "quantize.cuh"

namespace aircache {

namespace {

struct DecodeQParams {
    const float *k_scale, *v_scale;
    const int64_t *offsets;
    const int32_t *lens;
    const uint16_t *q;   // [items, heads of an item, D]
    float *out;          // the same
    int32_t *tickets;    // [items], zero between calls
    float *partials;     // [2 * CTAs][slot]
    uint32_t *status;
    int64_t rows, scale_blocks, first_region;
    int items, n_regions, split;   // split: KV heads per region where an item is a (region, head), else 1
    int row_heads;       // KV heads of a row in memory
    int Hq, G;           // query heads of an item, of a KV head
    float sl2;           // scale * log2(e)
};

constexpr int kTile = 32;               // rows of a warp's tile: two blocks of 16, the rows of an MMA and of a TMA box
constexpr int kBlocks = kTile / 16;
constexpr float kLift = 2048.f;   // of the weights, above fp16's subnormal numbers
// The largest V scale seen starts here, so that kLift over it is a number: over 2^-126, the scale of a block of zeros, it is
// not.  What the weights cannot hold then, 2^-36 * 2^-116 times a code of at most 448, is far below the smallest normal fp32 number.  (1 / scale, and kLift as a
// factor of every tile: 191.5 against 188.4 us for a batch of 64.)
constexpr float kLeastTop = 0x1p-116f;

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

// 16 bytes of shared memory, not asked for ahead of where the program has them (volatile): with 9 to 16 heads of 128 channels
// there are no registers for more of them at a time
__device__ __forceinline__ uint4 lds16(const void *from) {
    uint4 x;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(smem_u32(from)) : "memory");
    return x;
}

// the warps of one KV head
__device__ __forceinline__ void head_barrier(int head, int threads) {
    asm volatile("bar.sync %0, %1;" ::"r"(head + 1), "r"(threads) : "memory");
}

template <int D, int HEADS, int NT>
struct DecodeQCfg {
    static constexpr int WARPS = 8;
    static constexpr int SUBS = WARPS / HEADS;
    static constexpr int THREADS = WARPS * 32;
    static constexpr int CHUNKS = D / 64;                  // 64 channels of K: 16 per lane
    static constexpr int MT = D / 16;                      // channel tiles of O^T
    static constexpr int HALF = kTile * D;                 // bytes of a warp's tile of K or V
    static constexpr int STAGE = 2 * HALF;
    static constexpr int STAGES = D == 128 ? 3 : 6;
    static constexpr int RING = WARPS * STAGES * STAGE;
    static constexpr int BARS = WARPS * STAGES * 8;
    static constexpr int TABLES = (3 * kMaxRegions + 1) * 4;
    static constexpr int SMEM = 1024 + RING + BARS + TABLES;
    static_assert(MT * 4 * 32 * 4 <= STAGE, "a stage takes the sums of 8 heads");
    static_assert(SMEM <= 232448 - 2048, "shared memory of a block");
};

// An item stays whole up to this many tiles (of one head's warps) above the equal share: one image, 112 items of 27 tiles on
// average, 11.7 us whole and 15.6 with the longest ones cut (a merge takes as long as some 30 tiles).
constexpr int kWholeTiles = 32;

// a / b for a >= 0, b > 0, through the fp32 divider when both are below 2^23 (an integer division by a run-time divisor costs
// some hundred cycles of the plan)
__device__ __forceinline__ int small_div(int a, int b) {
    if (a >= (1 << 23) || b >= (1 << 23)) return a / b;
    int q = (int)__fdividef((float)a, (float)b);
    if (q * b > a) --q;
    if ((q + 1) * b <= a) ++q;
    return q;
}

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
__global__ void __launch_bounds__(DecodeQCfg<D, HEADS, NT>::THREADS, 1)
decode_quantized_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const DecodeQParams p) {
    using C = DecodeQCfg<D, HEADS, NT>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
    unsigned char *s_ring = smem;
    int *s_P = reinterpret_cast<int *>(smem + C::RING + C::BARS);   // [items + 1] first tile of an item
    int *s_off = s_P + kMaxRegions + 1, *s_len = s_off + kMaxRegions;
    __shared__ float4 s_state[C::WARPS * 4];   // references and sums of a warp's heads
    __shared__ int s_sum[C::WARPS], s_free[C::WARPS];
    __shared__ int s_last[2];   // items to be merged by this CTA: its last one, its first one
    __shared__ volatile int s_abort;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int head = warp % HEADS, sub = warp / HEADS;
    const uint32_t bars = smem_u32(smem + C::RING) + warp * (C::STAGES * 8);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0) {
        for (int i = 0; i < C::STAGES; ++i) mbar_init(bars + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 0) {
        s_abort = 0;
        s_last[0] = s_last[1] = -1;
        asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];" ::"l"(&tm_k), "l"(&tm_v) : "memory");
    }
    {   // asked into L2 ahead of the wait (no value is used): lengths, first rows, this block's share of the queries
        const int regions = p.n_regions;
        if (tid * 128 < regions * 4) prefetch_l2(reinterpret_cast<const char *>(p.lens) + tid * 128);
        if (tid * 128 < regions * 8) prefetch_l2(reinterpret_cast<const char *>(p.offsets) + tid * 128);
        const int64_t bytes = (int64_t)p.items * p.Hq * D * 2, at = ((int64_t)tid * gridDim.x + blockIdx.x) * 128;
        if (at < bytes) prefetch_l2(reinterpret_cast<const char *>(p.q) + at);
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // The CTA's tiles [t0, t1) and, of the item that they begin in: its number, first tile, end, first row, rows.
    const int cta = blockIdx.x;
    constexpr int RPL = 5;   // regions of a lane
    const bool pieces = p.items <= (int)gridDim.x && p.n_regions <= 32 * RPL;
    int t0, t1, item, item_first, item_end, item_off, n, c_first = 0, c_last = 0, lead_first = 0, lead_last = 0, total = 0, ctas = gridDim.x;
    if (pieces) {
        const int regions = p.n_regions, rpl = (regions + 31) / 32;
        int len[RPL], off[RPL], un[RPL], sum = 0, most = 0;
#pragma unroll
        for (int j = 0; j < RPL; ++j) {
            const int r = lane * rpl + j;
            len[j] = off[j] = 0;
            un[j] = -1;
            if (j < rpl && r < regions) {
                len[j] = rows_in_use(p.offsets, p.lens, r, p.rows, p.first_region, p.scale_blocks);
                off[j] = (int)p.offsets[r];
                un[j] = (len[j] + kTile - 1) / kTile;
                sum += un[j];
                most = max(most, un[j]);
            }
        }
        sum = __reduce_add_sync(0xffffffffu, sum) * p.split;
        most = __reduce_max_sync(0xffffffffu, most);
        const int share = max(small_div(sum + ctas - 1, ctas), 1);
        // the CTA's item: of which region (and where that is: its lane and slot), its first CTA, its pieces
        int found = -1, slot = 0, src, f_first, f_pieces = 1;
        if (most <= share + kWholeTiles / HEADS) {   // every item whole, in order
            if (cta >= p.items) return;
            found = p.split > 1 ? small_div(cta, p.split) : cta;
            src = rpl > 1 ? small_div(found, rpl) : found;
            slot = found - src * rpl;
            f_first = found * p.split;
        } else {
            int cap = max(most, 1);
            // pieces of an item of u tiles: one, or as many as pieces of `cap` tiles take
            auto pieces_of = [&](int u) { return u <= cap ? 1 : small_div(u + cap - 1, cap); };
            {   // the smallest of share, 9/8 of it, ... whose pieces find a CTA each
                for (cap = share; cap < most; cap += (cap + 7) / 8) {
                    int need = 0;
#pragma unroll
                    for (int j = 0; j < RPL; ++j)
                        if (j < rpl && un[j] >= 0) need += pieces_of(un[j]);
                    if ((int)__reduce_add_sync(0xffffffffu, need) * p.split <= ctas) break;
                }
            }
            int mine = 0, first = 0;
#pragma unroll
            for (int j = 0; j < RPL; ++j)
                if (j < rpl && un[j] >= 0) mine += pieces_of(un[j]);
            int run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += x;
            }
            run -= mine;
#pragma unroll
            for (int j = 0; j < RPL; ++j) {
                if (j >= rpl || un[j] < 0) continue;
                const int pc = pieces_of(un[j]);
                if (cta >= run * p.split && cta < (run + pc) * p.split) {
                    found = lane * rpl + j;
                    slot = j;
                    first = run * p.split;
                    f_pieces = pc;
                }
                run += pc;
            }
            const unsigned who = __ballot_sync(0xffffffffu, found >= 0);
            if (who == 0) return;
            src = __ffs(who) - 1;
            found = __shfl_sync(0xffffffffu, found, src);
            slot = __shfl_sync(0xffffffffu, slot, src);
            f_first = __shfl_sync(0xffffffffu, first, src);
            f_pieces = __shfl_sync(0xffffffffu, f_pieces, src);
        }
        item_end = n = item_off = 0;
#pragma unroll
        for (int j = 0; j < RPL; ++j)
            if (j == slot) { item_end = un[j]; n = len[j]; item_off = off[j]; }
        item_end = __shfl_sync(0xffffffffu, item_end, src);
        n = __shfl_sync(0xffffffffu, n, src);
        item_off = __shfl_sync(0xffffffffu, item_off, src);
        const int h = f_pieces == 1 ? cta - f_first : small_div(cta - f_first, f_pieces), piece = cta - f_first - h * f_pieces;
        item = found * p.split + h;
        c_first = f_first + h * f_pieces;
        c_last = c_first + f_pieces - 1;
        item_first = 0;
        t0 = (int)((int64_t)item_end * piece / f_pieces);
        t1 = (int)((int64_t)item_end * (piece + 1) / f_pieces);
        if (item_end == 0) {
            for (int e = tid; e < p.Hq * D; e += C::THREADS) p.out[(int64_t)item * p.Hq * D + e] = 0.f;
            return;
        }
    } else {
        // first tile, first row and rows of every item, THREADS of them at a time
        int base = 0;
        for (int at0 = 0; at0 < p.items; at0 += C::THREADS) {
            const int at = at0 + tid;
            int u = 0;
            if (at < p.items) {
                const int len = rows_in_use(p.offsets, p.lens, at, p.rows, p.first_region, p.scale_blocks);
                s_off[at] = (int)p.offsets[at];
                s_len[at] = len;
                u = (len + kTile - 1) / kTile;
            }
            int incl = u;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            if (lane == 31) s_sum[warp] = incl;
            __syncthreads();
            int before = base + incl - u;
#pragma unroll
            for (int w = 0; w < C::WARPS; ++w) {
                if (w < warp) before += s_sum[w];
                base += s_sum[w];
            }
            if (at < p.items) s_P[at] = before;
            __syncthreads();
        }
        if (tid == 0) s_P[p.items] = base;
        __syncthreads();
        total = s_P[p.items];
        for (int i = cta; i < p.items; i += gridDim.x)
            if (s_len[i] == 0)
                for (int e = tid; e < p.Hq * D; e += C::THREADS) p.out[(int64_t)i * p.Hq * D + e] = 0.f;
        ctas = min(ctas, total);   // each of them has a tile
        if (cta >= ctas) return;
        t0 = (int)((int64_t)total * cta / ctas);
        t1 = (int)((int64_t)total * (cta + 1) / ctas);
        item = find_item(s_P, p.items, t0);
        item_first = s_P[item];
        item_end = s_P[item + 1];
        item_off = s_off[item];
        n = s_len[item];
    }

    // the warp's tiles: tau = sub mod SUBS in [t0, t1); the ring is filled STAGES - 1 tiles ahead
    const uint32_t ring = smem_u32(s_ring) + warp * (C::STAGES * C::STAGE);
    int tau = t0 + (sub - t0 % C::SUBS + C::SUBS) % C::SUBS, stage = 0;
    uint32_t parity = 0;
    int ask = tau, ask_stage = 0, ask_item = item, ask_first = item_first, ask_end = item_end, ask_off = item_off, ask_n = n;
    int ask_region = pieces ? item / p.split : item;
    const int ask_head = p.split > 1 ? item - ask_region * p.split : head;   // (only pieces are of one head)
    // places of the scales of the tiles in the ring, the next one first.  (Places, not values: a move of a value that is being
    // loaded waits for it.)  A tile's scales are loaded while the one before it is worked on.
    int scale_at[C::STAGES];
    const float *const k_scales = p.k_scale + p.first_region * p.row_heads, *const v_scales = p.v_scale + p.first_region * p.row_heads;
    auto issue = [&](int &place) {
        place = 0;
        if (ask < t1) {
            if (ask >= ask_end) {   // (a list of items only: a piece ends with its item or before)
                while (ask >= s_P[ask_item + 1]) ++ask_item;
                ask_region = ask_item;
                ask_first = s_P[ask_item];
                ask_end = s_P[ask_item + 1];
                ask_off = s_off[ask_item];
                ask_n = s_len[ask_item];
            }
            const int row0 = (ask - ask_first) * kTile;
            if (lane == 0) {   // (the item's last tile may need one block only)
                const uint32_t bar = bars + 8 * ask_stage, dst = ring + ask_stage * C::STAGE;
                const bool both = row0 + 16 < ask_n;
                mbar_expect_tx(bar, both ? C::STAGE : C::STAGE / 2);
                tma_load_3d(dst, &tm_k, 0, ask_head, ask_off + row0, bar);
                if (both) tma_load_3d(dst + 16 * D, &tm_k, 0, ask_head, ask_off + row0 + 16, bar);
                tma_load_3d(dst + C::HALF, &tm_v, 0, ask_head, ask_off + row0, bar);
                if (both) tma_load_3d(dst + C::HALF + 16 * D, &tm_v, 0, ask_head, ask_off + row0 + 16, bar);
            }
            place = (ask_off / kScaleRows + row0 / kScaleRows + ask_region) * p.row_heads + ask_head;
            ask += C::SUBS;
        }
        ask_stage = ask_stage + 1 == C::STAGES ? 0 : ask_stage + 1;
    };
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) issue(scale_at[i]);
    float next_k_scale = k_scales[scale_at[0]], next_v_scale = v_scales[scale_at[0]];

    // an item's queries as they are: asked for while the item before is put together
    uint32_t q_raw[NT][C::CHUNKS][8];
    auto load_q = [&](int of) {
        const uint16_t *from = p.q + ((int64_t)of * p.Hq + head * p.G) * D + t * (D / 4);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (nt * 8 + g < p.G) x = *reinterpret_cast<const uint4 *>(from + (nt * 8 + g) * D + c * 16 + i * 8);
                    q_raw[nt][c][4 * i] = x.x;
                    q_raw[nt][c][4 * i + 1] = x.y;
                    q_raw[nt][c][4 * i + 2] = x.z;
                    q_raw[nt][c][4 * i + 3] = x.w;
                }
    };
    load_q(item);

    bool ok = true;
    while (true) {
        const int end = min(t1, item_end);

        // the item's queries as fp16 fragments: columns are the heads of the KV group, lane (g, t) holds head g (+ 8)
        uint32_t qf[NT][C::CHUNKS][8];
        float f[NT][2];   // logits of heads 2t, 2t + 1 (+ 8) from the products, without the K scale
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            uint32_t top2 = 0;
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c)
#pragma unroll
                for (int a = 0; a < 8; ++a) top2 = __vmaxu2(top2, q_raw[nt][c][a] & 0x7fff7fffu);
            uint32_t top = max(top2 & 0xffffu, top2 >> 16);
            if (top >= 0x7f80) {   // infinities and NaN do not count
                top = 0;
#pragma unroll
                for (int c = 0; c < C::CHUNKS; ++c)
#pragma unroll
                    for (int a = 0; a < 8; ++a) {
                        const uint32_t l = q_raw[nt][c][a] & 0x7fffu, u = q_raw[nt][c][a] >> 16 & 0x7fffu;
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
                for (int a = 0; a < 8; ++a) qf[nt][c][a] = f16x2(bf16lo(q_raw[nt][c][a]) * up, bf16hi(q_raw[nt][c][a]) * up);
            f[nt][0] = __shfl_sync(0xffffffffu, down, 8 * t) * p.sl2;
            f[nt][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4) * p.sl2;
        }

        float acc[NT][C::MT][4], ref[NT][2], sum[NT][2], v_top = kLeastTop, v_inv = kLift / kLeastTop;
        bool unset[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < C::MT; ++c) acc[nt][c][0] = acc[nt][c][1] = acc[nt][c][2] = acc[nt][c][3] = 0.f;
            ref[nt][0] = ref[nt][1] = 0.f;   // none yet: the first finite logits set it
            unset[nt][0] = unset[nt][1] = true;
            sum[nt][0] = sum[nt][1] = 0.f;
        }

        for (; tau < end; tau += C::SUBS) {
            if (ok) ok = mbar_wait(bars + 8 * stage, parity, &s_abort, p.status, 10);
            if (!__all_sync(0xffffffffu, ok)) {   // given up: what is written is incomplete, and reported
                ok = false;
                continue;
            }
            issue(scale_at[C::STAGES - 1]);
            const unsigned char *tile = s_ring + (warp * C::STAGES + stage) * C::STAGE;
            const float k_scale = next_k_scale, v_scale = next_v_scale;
#pragma unroll
            for (int i = 0; i + 1 < C::STAGES; ++i) scale_at[i] = scale_at[i + 1];
            next_k_scale = k_scales[scale_at[0]];
            next_v_scale = v_scales[scale_at[0]];
            if (++stage == C::STAGES) { stage = 0; parity ^= 1; }

            const int rows = n - (tau - item_first) * kTile;   // of the tile, kTile or more unless it is the item's last
            float x[kBlocks][NT][4];   // logits (log2) above the reference
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                float s[NT][2][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nt][0][i] = s[nt][1][i] = 0.f;
                const unsigned char *k_tile = tile + b * 16 * D;
#pragma unroll
                for (int c = 0; c < C::CHUNKS; ++c) {
                    // 128 channels: rows of 128 bytes, 16-byte piece i of row r at i ^ (r & 7); eight lanes read pieces 2t (or 2t + 1)
                    // of two rows that differ in the lowest bit: all banks once.  64: rows of 64 bytes, piece i at i ^ (r / 2 & 3).
                    const int at = D == 128 ? g * 128 + (((2 * t + c) ^ g) & 7) * 16 : g * 64 + ((t ^ (g >> 1)) & 3) * 16;
                    const uint4 ka = *reinterpret_cast<const uint4 *>(k_tile + at), kb = *reinterpret_cast<const uint4 *>(k_tile + 8 * D + at);
                    const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t a0 = e4m3x2_f16x2(wa[w] & 0xffffu), a2 = e4m3x2_f16x2(wa[w] >> 16);
                        const uint32_t a1 = e4m3x2_f16x2(wb[w] & 0xffffu), a3 = e4m3x2_f16x2(wb[w] >> 16);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            mma_f16_16816(s[nt][w & 1], a0, a1, a2, a3, qf[nt][c][2 * w], qf[nt][c][2 * w + 1]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[b][nt][i] = fmaf(s[nt][0][i] + s[nt][1][i], f[nt][i & 1] * k_scale, -ref[nt][i & 1]);
            }
            if (rows < kTile) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (16 * b + g >= rows) x[b][nt][0] = x[b][nt][1] = -INFINITY;
                        if (16 * b + g + 8 >= rows) x[b][nt][2] = x[b][nt][3] = -INFINITY;
                    }
            }
            float tops[NT][2];   // of this lane's keys
            bool moves = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    tops[nt][j] = fmaxf(x[0][nt][j], x[0][nt][j + 2]);
#pragma unroll
                    for (int b = 1; b < kBlocks; ++b) tops[nt][j] = fmaxf(tops[nt][j], fmaxf(x[b][nt][j], x[b][nt][j + 2]));
                    moves = moves || unset[nt][j] || tops[nt][j] > 4.f;
                }
            if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float top = tops[nt][j];
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                        const bool sets = unset[nt][j] && top > -INFINITY;
                        const float now = ref[nt][j] + (sets ? top : unset[nt][j] ? 0.f : fmaxf(top, 0.f));
                        const float up = now - ref[nt][j], shrink = sets ? 0.f : fast_exp2(-up);   // (by what the reference really moves)
                        unset[nt][j] = unset[nt][j] && !sets;
                        ref[nt][j] = now;
#pragma unroll
                        for (int b = 0; b < kBlocks; ++b) {
                            x[b][nt][j] -= up;
                            x[b][nt][j + 2] -= up;
                        }
                        sum[nt][j] *= shrink;
#pragma unroll
                        for (int c = 0; c < C::MT; ++c) {
                            acc[nt][c][j] *= shrink;
                            acc[nt][c][j + 2] *= shrink;
                        }
                    }
            }
            if (v_scale > v_top) {   // (all lanes alike)
                const float shrink = v_top / v_scale;
                v_top = v_scale;
                v_inv = kLift / v_scale;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < C::MT; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[nt][c][i] *= shrink;
            }
            const float vf = v_scale * v_inv;
            // Both blocks of a tile at a time, or one (9 to 16 heads: the registers).
            constexpr int GROUP = NT == 2 ? 1 : kBlocks;
#pragma unroll
            for (int b0 = 0; b0 < kBlocks; b0 += GROUP) {
                uint32_t head_b[GROUP][NT][2], rest_b[GROUP][NT][2], vw[GROUP][4][C::MT / 2];
#pragma unroll
                for (int b = 0; b < GROUP; ++b) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {   // keys g (i = 0) and g + 8
                            const float p0 = fast_exp2(x[b0 + b][nt][2 * i]), p1 = fast_exp2(x[b0 + b][nt][2 * i + 1]);
                            sum[nt][0] += p0;
                            sum[nt][1] += p1;
                            const uint32_t hi = f16x2(p0 * vf, p1 * vf);
                            const float2 back = f16x2_f32(hi);
                            head_b[b][nt][i] = movmatrix_trans(hi);
                            rest_b[b][nt][i] = movmatrix_trans(f16x2(fmaf(p0, vf, -back.x), fmaf(p1, vf, -back.y)));
                        }
                    const unsigned char *v_tile = tile + C::HALF + (b0 + b) * 16 * D;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = 2 * t + (i & 1) + 8 * (i >> 1);
                        if (D == 128) {
                            const unsigned char *from = v_tile + key * 128 + ((g ^ key) & 7) * 16;
                            const uint4 x4 = NT == 2 ? lds16(from) : *reinterpret_cast<const uint4 *>(from);
                            vw[b][i][0] = x4.x; vw[b][i][1] = x4.y; vw[b][i][C::MT / 2 - 2] = x4.z; vw[b][i][C::MT / 2 - 1] = x4.w;
                        } else {
                            const uint2 x2 = *reinterpret_cast<const uint2 *>(v_tile + key * 64 + (((g >> 1) ^ (key >> 1)) & 3) * 16 + (g & 1) * 8);
                            vw[b][i][0] = x2.x; vw[b][i][1] = x2.y;
                        }
                    }
                    if (rows < kTile) {   // behind the rows in use: whatever lies there
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * (b0 + b) + 2 * t + (i & 1) + 8 * (i >> 1) >= rows) {
#pragma unroll
                                for (int w = 0; w < C::MT / 2; ++w) vw[b][i][w] = 0;
                            }
                    }
                }
                // The products of a tile are summed from zero and added to the sums by the FMA pipe: the tensor core cuts off what an
                // addition leaves beyond 24 bits, and over hundreds of rows of one warp that adds up (4300 rows: 6.3e-6 of the
                // output, 2.7e-7 this way; 184 -> 188 us for a batch of 64; with 16 heads to each of two KV heads and some 150 bytes of
                // spills, eight sequences of 1139 rows 44.3 -> 49.8, 32 of them 124 -> 139).
#pragma unroll
                for (int w = 0; w < C::MT / 2; ++w) {
                    uint32_t a[GROUP][8];   // channels 4w..4w+3 of this lane's stretch, two keys abreast
#pragma unroll
                    for (int b = 0; b < GROUP; ++b) {
                        const uint32_t l01 = __byte_perm(vw[b][0][w], vw[b][1][w], 0x5140), u01 = __byte_perm(vw[b][0][w], vw[b][1][w], 0x7362);
                        const uint32_t l23 = __byte_perm(vw[b][2][w], vw[b][3][w], 0x5140), u23 = __byte_perm(vw[b][2][w], vw[b][3][w], 0x7362);
                        a[b][0] = e4m3x2_f16x2(l01 & 0xffffu);
                        a[b][1] = e4m3x2_f16x2(l01 >> 16);
                        a[b][2] = e4m3x2_f16x2(l23 & 0xffffu);
                        a[b][3] = e4m3x2_f16x2(l23 >> 16);
                        a[b][4] = e4m3x2_f16x2(u01 & 0xffffu);
                        a[b][5] = e4m3x2_f16x2(u01 >> 16);
                        a[b][6] = e4m3x2_f16x2(u23 & 0xffffu);
                        a[b][7] = e4m3x2_f16x2(u23 >> 16);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float low[4] = {0.f, 0.f, 0.f, 0.f}, high[4] = {0.f, 0.f, 0.f, 0.f};   // channel tiles 2w and 2w + 1
#pragma unroll
                        for (int b = 0; b < GROUP; ++b) {
                            mma_f16_16816(low, a[b][0], a[b][1], a[b][2], a[b][3], rest_b[b][nt][0], rest_b[b][nt][1]);
                            mma_f16_16816(high, a[b][4], a[b][5], a[b][6], a[b][7], rest_b[b][nt][0], rest_b[b][nt][1]);
                            mma_f16_16816(low, a[b][0], a[b][1], a[b][2], a[b][3], head_b[b][nt][0], head_b[b][nt][1]);
                            mma_f16_16816(high, a[b][4], a[b][5], a[b][6], a[b][7], head_b[b][nt][0], head_b[b][nt][1]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const float2 l = add2(make_float2(acc[nt][2 * w][i], acc[nt][2 * w][i + 1]), make_float2(low[i], low[i + 1]));
                            const float2 h = add2(make_float2(acc[nt][2 * w + 1][i], acc[nt][2 * w + 1][i + 1]), make_float2(high[i], high[i + 1]));
                            acc[nt][2 * w][i] = l.x;
                            acc[nt][2 * w][i + 1] = l.y;
                            acc[nt][2 * w + 1][i] = h.x;
                            acc[nt][2 * w + 1][i + 1] = h.y;
                        }
                    }
                }
            }
            __syncwarp();   // (the stage may be refilled from the next tile on)
        }

        int next = item;   // (a list of items: empty ones are passed over)
        if (item_end < t1) {
            do ++next; while (s_P[next + 1] <= item_end);
            load_q(next);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (unset[nt][j]) ref[nt][j] = -INFINITY;
        // the end of the item's part: sums over the lanes of a head, true units; then the warps of a head put their states
        // into the ring stages that they have just read and share out the channels of the merged one
        const bool whole = item_first >= t0 && item_end <= t1;
        const int64_t slot_floats = partial_slot_floats(p.Hq, D);
        float *slot = p.partials + (2 * (int64_t)cta + (item_first >= t0 ? 1 : 0)) * slot_floats;
        float *item_out = whole ? p.out + (int64_t)item * p.Hq * D : slot;
        const float unit = v_top * (1.f / kLift);
        const int free_stage = (stage + C::STAGES - 1) % C::STAGES;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], 4);
                sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], 8);
                sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], 16);
            }
            float weight[C::SUBS][2], top[2] = {ref[nt][0], ref[nt][1]}, all[2] = {sum[nt][0], sum[nt][1]};
            const float *posted[C::SUBS];
            weight[0][0] = weight[0][1] = 1.f;
            if (C::SUBS > 1) {
                float *post = reinterpret_cast<float *>(s_ring + (warp * C::STAGES + free_stage) * C::STAGE) + lane;
#pragma unroll
                for (int c = 0; c < C::MT; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) post[(c * 4 + i) * 32] = acc[nt][c][i] * unit;
                if (g == 0) s_state[warp * 4 + t] = make_float4(top[0], top[1], all[0], all[1]);
                if (lane == 0) s_free[warp] = free_stage;
                head_barrier(head, C::SUBS * 32);
                top[0] = top[1] = -1e30f;
#pragma unroll
                for (int i = 0; i < C::SUBS; ++i) {
                    const float4 x = s_state[(i * HEADS + head) * 4 + t];
                    weight[i][0] = x.x;
                    weight[i][1] = x.y;
                    top[0] = fmaxf(top[0], x.x);
                    top[1] = fmaxf(top[1], x.y);
                }
                all[0] = all[1] = 0.f;
#pragma unroll
                for (int i = 0; i < C::SUBS; ++i) {
                    const int w = i * HEADS + head;
                    const float4 x = s_state[w * 4 + t];
                    posted[i] = reinterpret_cast<const float *>(s_ring + (w * C::STAGES + s_free[w]) * C::STAGE) + lane;
#pragma unroll
                    for (int j = 0; j < 2; ++j) weight[i][j] = fast_exp2(weight[i][j] - top[j]);
                    all[0] = fmaf(x.z, weight[i][0], all[0]);
                    all[1] = fmaf(x.w, weight[i][1], all[1]);
                }
            }
            float times[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) times[j] = !whole ? 1.f : all[j] > 0.f || all[j] != all[j] ? 1.f / all[j] : 0.f;
#pragma unroll
            for (int c = 0; c < C::MT; ++c) {
                if (C::SUBS > 1 && c % C::SUBS != sub) continue;
                float m[4];
                if (C::SUBS > 1) {
                    m[0] = m[1] = m[2] = m[3] = 0.f;
#pragma unroll
                    for (int i = 0; i < C::SUBS; ++i)
#pragma unroll
                        for (int x = 0; x < 4; ++x) m[x] = fmaf(posted[i][(c * 4 + x) * 32], weight[i][x & 1], m[x]);
                } else {
#pragma unroll
                    for (int x = 0; x < 4; ++x) m[x] = acc[nt][c][x] * unit;
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (nt * 8 + 2 * t + j < p.G)
                        *reinterpret_cast<float2 *>(item_out + (int64_t)(head * p.G + nt * 8 + 2 * t + j) * D + g * (D / 8) + 2 * c) =
                            make_float2(m[j] * times[j], m[j + 2] * times[j]);
            }
            if (!whole && g == 0 && sub == 0) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int h = nt * 8 + 2 * t + j;
                    if (h >= p.G) continue;
                    slot[(int64_t)p.Hq * D + head * p.G + h] = top[j];
                    slot[(int64_t)p.Hq * (D + 1) + head * p.G + h] = all[j];
                }
            }
            if (C::SUBS > 1) {   // the stages go back to the copies
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                head_barrier(head, C::SUBS * 32);
            }
        }
        if (!whole) {
            if (!pieces) {   // the CTAs that have a part of the item, in order: tile u belongs to CTA ((u + 1) * ctas - 1) / total
                c_first = (int)(((int64_t)(item_first + 1) * ctas - 1) / total);
                c_last = (int)(((int64_t)item_end * ctas - 1) / total);
            }
            __syncthreads();
            const bool leads = item_end < t1;   // the end of an item that began before this CTA's part
            if (tid == 0) {
                __threadfence();
                s_last[leads] = atomicAdd(p.tickets + item, 1) == c_last - c_first ? item : -1;
                __threadfence();
            }
            if (leads) {   // whether it was the last one is looked at in the end
                lead_first = c_first;
                lead_last = c_last;
            }
        }
        if (item_end >= t1) break;
        item = next;
        item_first = item_end;
        item_end = s_P[item + 1];
        n = s_len[item];
    }
    // the items whose last part was this CTA's are merged
    __syncthreads();
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const int item = s_last[which];
        if (item < 0) continue;
        const int c0 = which ? lead_first : c_first, c1 = which ? lead_last : c_last;
        const int64_t slot_floats = partial_slot_floats(p.Hq, D);
        for (int e = tid; e < p.Hq * D / 4; e += C::THREADS) {   // (four channels a thread: one element each took a trip to L2 after the other)
            const int hq = e / (D / 4);
            float m = -1e30f, l = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int c = c0; c <= c1; ++c) {
                const float *from = p.partials + (2 * (int64_t)c + (c == c0 ? 1 : 0)) * slot_floats;
                const float cm = __ldcg(from + (int64_t)p.Hq * D + hq), cl = __ldcg(from + (int64_t)p.Hq * (D + 1) + hq);
                const float4 co = __ldcg(reinterpret_cast<const float4 *>(from) + e);
                const float now = fmaxf(m, cm), mine = fast_exp2(m - now), theirs = fast_exp2(cm - now);
                m = now;
                l = l * mine + cl * theirs;
                o.x = o.x * mine + co.x * theirs;
                o.y = o.y * mine + co.y * theirs;
                o.z = o.z * mine + co.z * theirs;
                o.w = o.w * mine + co.w * theirs;
            }
            const float times = l > 0.f || l != l ? 1.f / l : 0.f;
            reinterpret_cast<float4 *>(p.out + (int64_t)item * p.Hq * D)[e] = make_float4(o.x * times, o.y * times, o.z * times, o.w * times);
        }
        if (tid == 0) p.tickets[item] = 0;
    }
    // a wait that gave up: copies in flight get their time before the block's memory goes
    if (s_abort)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

// e4m3 [rows, heads, D] as a 3-D tensor of bytes (D, heads, rows); a box is 16 rows of one head.
int make_map(CUtensorMap *tm, const void *base, int D, int heads, int64_t rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) { set_last_cuda_error(cudaErrorSymbolNotFound); return AIRCACHE_ERR_CUDA; }
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)D, (cuuint64_t)heads * D};
    const cuuint32_t box[3] = {(cuuint32_t)D, 1, 16}, estr[3] = {1, 1, 1};
    const CUresult rc = fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(base), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (rc != CUDA_SUCCESS) { set_last_cuda_error(cudaErrorInvalidValue); return AIRCACHE_ERR_CUDA; }
    return AIRCACHE_OK;
}

struct Maps { CUtensorMap k, v; };

template <int D, int HEADS, int NT>
int launch_t(const Maps &m, const DecodeQParams &p, int ctas, int dev, cudaStream_t st) {
    using C = DecodeQCfg<D, HEADS, NT>;
    static std::atomic<uint64_t> allowed[kMaxDevices];
    const int rc = allow_shared_memory((const void *)decode_quantized_kernel<D, HEADS, NT>, C::SMEM, dev, allowed);
    if (rc) return rc;
    return launch_dependent(decode_quantized_kernel<D, HEADS, NT>, dim3(ctas), dim3(C::THREADS), C::SMEM, st, m.k, m.v, p);
}

template <int D, int HEADS>
int launch_g(const Maps &m, const DecodeQParams &p, int ctas, int dev, cudaStream_t st) {
    return p.G > 8 ? launch_t<D, HEADS, 2>(m, p, ctas, dev, st) : launch_t<D, HEADS, 1>(m, p, ctas, dev, st);
}

template <int D>
int launch_d(const Maps &m, const DecodeQParams &p, int heads, int ctas, int dev, cudaStream_t st) {
    switch (heads) {
        case 1: return launch_g<D, 1>(m, p, ctas, dev, st);
        case 2: return launch_g<D, 2>(m, p, ctas, dev, st);
        case 4: return launch_g<D, 4>(m, p, ctas, dev, st);
        case 8: return launch_g<D, 8>(m, p, ctas, dev, st);
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
    p.k_scale = c->k_scale;
    p.v_scale = c->v_scale;
    p.offsets = c->offsets;
    p.lens = c->lens;
    p.q = static_cast<const uint16_t *>(q);
    p.out = out;
    p.tickets = ws_ptr<int32_t>(ws, w.tickets);
    p.partials = ws_ptr<float>(ws, w.partials);
    p.status = ws_ptr<uint32_t>(ws, w.status);
    p.rows = c->total_rows;
    p.scale_blocks = c->scale_blocks;
    p.first_region = c->first_region;
    p.row_heads = row_heads_of(s);
    p.G = s->n_q_heads / s->n_kv_heads;
    p.items = (int)n_cells(s);
    p.n_regions = p.items;
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
    Maps m;
    if ((rc = make_map(&m.k, c->k, s->head_dim, p.row_heads, c->total_rows))) return rc;
    if ((rc = make_map(&m.v, c->v, s->head_dim, p.row_heads, c->total_rows))) return rc;
    return s->head_dim == 64 ? launch_d<64>(m, p, heads, ctas, dev, st) : launch_d<128>(m, p, heads, ctas, dev, st);
}

}  // namespace aircache
