// aircache_prompt_attn: causal attention of one layer over packed prompts, on the fifth-generation tensor cores.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp2(scale log2(e) <q_i, k_j> - ref_i)
//
// Bound by the tensor core (4 d flop per query head, query and visible key) and, next to it, by the exponentials: an SM
// multiplies a 128 x 128 x 128 tile in some 512 cycles and takes 16384 exponentials, one per logit, in 1024.
//
// Work.  The G query heads of a KV group read the same keys, so rows of a tile are (token, head of the group) pairs, the
// head inside: 128 / G tokens (rounded down) of all G heads, 126 rows at G = 7.  A tile then spans few tokens, which keeps the part
// that the causal mask throws away small, and a turn of a few tokens still fills rows.  A block takes two such tiles, one behind
// the other, of one sequence and KV head, and goes over the keys in tiles of 128, all of them once.  Blocks are numbered from the
// last tokens of the last sequence on, so that within a sequence those with the most keys start first (sequences go by their number,
// not by their length); a block that is done takes the work of one that
// has not started (cluster launch control), so that its first copies and products run beside the end of the unit before
// (9338 tokens and 64 heads: 1327 -> 1245 us when it came).  In calls of so few blocks that each has an SM of its own, a block takes one
// row tile and its two halves share the key tiles, even and odd; their sums meet in the end.
//
// Roles.  Warp 8: TMA producer, Q once, then K and V tiles through one ring.  Warp 9: one thread issues the MMAs: S_i = Q_i K^T
// (M = 128 rows, N = 128 keys, both operands from shared memory, K-major) and O_i += P_i V (P_i from tensor memory, V with
// the keys as the outer axis).  Warps 0-3 and 4-7: the softmax of tile 0 and 1, a thread a row, no exchange between
// threads: S_i from tensor memory, exponentials, P_i in bf16 back over the columns of S_i.  While one tile's softmax runs, the
// tensor core has the other tile's products.  MMAs of one thread are executed in order, so S_i of the next key tile is issued right behind
// the product that reads P_i.
//
// Measured (one B200, 1662 TFLOP/s by the library's own large products): 9338 tokens, 64 / 8 heads of 128, causal (1429 GFLOP) 1140 to
// 1190 us a call, 1356 to 1375 in a second of calls back to back, where the power cap holds the clock; eight prompts of 300 to 3172
// tokens, 28 / 4 heads (95 GFLOP) 132 and 144; 640 tokens of a small model 10.  A step (128 keys, two row tiles) takes 3500 to 3900
// cycles: its products alone 2900, since a product with A in shared memory takes 106 cycles where its arithmetic takes 64 (A in tensor
// memory: 75); a row tile's softmax 2500, of which the other tile's products cover most.  Not kept: two threads a row, steps of
// 64 keys with two score buffers, exponentials as polynomials, the weights handed over in halves (all slower).
//
// The reference of a row moves only when a logit is more than 2^16 above it (weights are floating-point numbers: it
// need not be the maximum); then its warp rescales O_i in tensor memory, behind the last product's commit.  Sums and O_i in fp32.  P is rounded to bf16 for the second
// product (up to 2^-8 of a weight, averaged over the keys, beside up to 2^-8 for the rounding of the output; both operands of a product have
// one type).  Off by 1.2 to 1.4 times what a 32-bit form with the same output is off by.
//
// The last key tile of a sequence may hold rows of the next one or of nothing: their logits are masked, and the V rows are
// zeroed in shared memory before they are multiplied (0 * NaN).
#include <cuda.h>

#include <atomic>
#include <mutex>

#include "common.cuh"
#include "ptx.cuh"

namespace aircache {

namespace {

__device__ uint32_t g_prompt_timeouts;   // blocks in which a bounded wait gave up, since the context was made

constexpr int kKeys = 128;             // keys of a tile
constexpr float kRise = 16.f;          // a row's reference moves when a logit is more than this above it (log2)

struct PromptParams {
    const int32_t *q_offsets, *k_offsets;
    char *out;
    int64_t out_token, out_head;   // bytes
    int n_seqs, q_tokens, k_tokens, n_kv_heads, G, tokens_per_tile, units, causal;
    float sl2;
};

// A block's unit of work: row tiles of one sequence and KV head.
struct Unit {
    int q0, n_q, k0, n_k;   // the sequence's rows
    int first, group;       // first token of the first tile; KV head, -1: no more units
    int split;              // one row tile, whose key tiles the two halves of the block share: even ones, odd ones
    int tiles[2];           // key tiles of each half
};

template <int D>
struct PromptCfg {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE = kKeys * D * 2;           // bytes of a Q, K or V tile
    static constexpr int HALF = kKeys * 128;             // of 64 channels of it
    static constexpr int SLOTS = D == 128 ? 5 : 8;
    static constexpr int SMEM = 1024 + (2 + SLOTS) * TILE;
    static constexpr int THREADS = 384;                  // three warpgroups of 168 registers a thread, moved below
};

// Matrix descriptors (umma_desc_sw128) as their two words: the upper one is the same for every tile here (groups of 8 rows
// 1024 bytes apart, version, 128-byte swizzle), the lower one is the start address in units of 16 bytes and, for a tile whose
// rows are the K axis (V), the distance to the next 64 elements of N.  One thread issues some 24 products in a thousand
// cycles: with the whole descriptor built for each of them that took it 2500.
constexpr uint32_t kDescHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_low(uint32_t smem_addr) { return smem_addr >> 4 | 1u << 16; }
__device__ __forceinline__ uint32_t desc_low_rows_are_k(uint32_t smem_addr) { return smem_addr >> 4 | (uint32_t)(kKeys * 128 >> 4) << 16; }

// D[tmem] (+)= A[smem] B[smem]^T, bf16, one step of 16 of the K axis
__device__ __forceinline__ void mma_smem(uint32_t tmem_d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 a, b;\nmov.b64 a, {%1, %4};\nmov.b64 b, {%2, %4};\nsetp.ne.b32 p, %5, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n"
        ::"r"(tmem_d), "r"(a), "r"(b), "r"(idesc), "r"(kDescHigh), "r"((uint32_t)accumulate) : "memory");
}
// the same with A in tensor memory
__device__ __forceinline__ void mma_tmem(uint32_t tmem_d, uint32_t tmem_a, uint32_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 b;\nmov.b64 b, {%2, %4};\nsetp.ne.b32 p, %5, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n"
        ::"r"(tmem_d), "r"(tmem_a), "r"(b), "r"(idesc), "r"(kDescHigh), "r"((uint32_t)accumulate) : "memory");
}
// 16 columns of this thread's lane as they are
#define AIRCACHE_R16(c, r) c(r[0]), c(r[1]), c(r[2]), c(r[3]), c(r[4]), c(r[5]), c(r[6]), c(r[7]), \
    c(r[8]), c(r[9]), c(r[10]), c(r[11]), c(r[12]), c(r[13]), c(r[14]), c(r[15])
__device__ __forceinline__ void tmem_st16_bits(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), AIRCACHE_R16("r", r) : "memory");
}
__device__ __forceinline__ void tmem_ld16_bits(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : AIRCACHE_R16("=r", r) : "r"(taddr) : "memory");
}
#undef AIRCACHE_R16

// 16 columns of tensor memory times `shrink`.
__device__ __forceinline__ void rescale16(uint32_t at, float shrink) {
    uint32_t r[16];
    tmem_ld16_bits(at, r);
#pragma unroll
    for (int e = 0; e < 16; ++e)
        r[e] = __float_as_uint(__uint_as_float(r[e]) * shrink);
    tmem_st16_bits(at, r);
    tmem_st_wait();
}

// Asks for a block of this grid that has not started yet; the answer (16 bytes) is counted on an mbarrier.
__device__ __forceinline__ void take_block(uint32_t answer, uint32_t bar) {
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(answer), "r"(bar) : "memory");
}
// The block of the answer, or -1 if there is none left.
__device__ __forceinline__ int taken_block(uint32_t answer) {
    uint32_t ok, x;
    asm volatile(
        "{\n.reg .b128 r;\n.reg .pred p;\n.reg .b32 y, z, w;\n"
        "ld.shared.b128 r, [%2];\n"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n"
        "mov.b32 %1, 0;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, r;\n}\n"
        : "=r"(ok), "=r"(x) : "r"(answer) : "memory");
    return ok ? (int)x : -1;
}

// ROW_TILES = 1: a unit has one row tile, whose key tiles the halves of the block share (split units).
template <int D, int ROW_TILES>
__global__ void __launch_bounds__(PromptCfg<D>::THREADS, 1)
prompt_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
              const __grid_constant__ CUtensorMap tm_v, const PromptParams p) {
    using C = PromptCfg<D>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ uint64_t s_bars[2 + 2 * C::SLOTS + 6 + 6];
    __shared__ __align__(16) uint32_t s_answer[4];
    __shared__ Unit s_unit[2];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    __shared__ uint32_t s_status;   // which wait gave up
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t q_smem = smem, ring = smem + 2 * C::TILE;
    const uint32_t bars = smem_u32(s_bars);
    const uint32_t q_full = bars, q_empty = bars + 8, kv_full = bars + 16, kv_empty = kv_full + 8 * C::SLOTS,
                   s_full = kv_empty + 8 * C::SLOTS, p_full = s_full + 16, o_done = p_full + 16, unit_full = o_done + 16,
                   unit_empty = unit_full + 16, answered = unit_empty + 16, met_all = answered + 8;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int TPT = p.tokens_per_tile;
    uint32_t *status = &s_status;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 9) tmem_alloc(smem_u32(&s_tmem), 512);
    if (warp == 8 && lane == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        for (int i = 0; i < C::SLOTS; ++i) {
            mbar_init(kv_full + 8 * i, 1);
            mbar_init(kv_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 128);
            mbar_init(o_done + 8 * i, 1);
            mbar_init(unit_full + 8 * i, 1);
            mbar_init(unit_empty + 8 * i, 9);   // a lane of each warp that reads a unit
        }
        mbar_init(answered, 1);
        mbar_init(met_all, 256);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_abort = 0;
        asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];\nprefetch.tensormap [%2];"
                     ::"l"(&tm_q), "l"(&tm_k), "l"(&tm_v) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    // The unit of turn `it`, as the producer has left it.
    auto next_unit = [&](int it, Unit &u) {
        const bool ok = __all_sync(0xffffffffu, mbar_wait(unit_full + 8 * (it & 1), it >> 1 & 1, &s_abort, status, 8));
        if (!ok) return false;
        u = s_unit[it & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(unit_empty + 8 * (it & 1));
        return u.group >= 0;
    };

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 8) {
            int block = blockIdx.x, slot = 0, loaded = 0, full_units = 0;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                Unit u = {};
                u.group = -1;
                if (block >= 0) {   // the block's unit: counted from the last one back
                    const int unit = p.units - 1 - block / p.n_kv_heads;
                    u.group = block % p.n_kv_heads;
                    int before = 0;
                    for (int s0 = 0; s0 < p.n_seqs && before <= unit; s0 += 32) {
                        const int s = s0 + lane;
                        int q0 = 0, n_q = 0, n = 0;
                        if (s < p.n_seqs) {
                            q0 = min(max(p.q_offsets[s], 0), p.q_tokens);
                            n_q = min(max(p.q_offsets[s + 1], q0), p.q_tokens) - q0;
                            n = (n_q + ROW_TILES * TPT - 1) / (ROW_TILES * TPT);
                        }
                        int incl = n;
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const int x = __shfl_up_sync(0xffffffffu, incl, o);
                            if (lane >= o) incl += x;
                        }
                        const int mine = before + incl - n;
                        const unsigned who = __ballot_sync(0xffffffffu, unit >= mine && unit < mine + n);
                        if (who) {
                            const int src = __ffs(who) - 1, at = s0 + src;
                            u.q0 = __shfl_sync(0xffffffffu, q0, src);
                            u.n_q = __shfl_sync(0xffffffffu, n_q, src);
                            u.first = (unit - __shfl_sync(0xffffffffu, mine, src)) * ROW_TILES * TPT;
                            u.k0 = min(max(p.k_offsets[at], 0), p.k_tokens);
                            u.n_k = min(max(p.k_offsets[at + 1], u.k0), p.k_tokens) - u.k0;
                        }
                        before += __shfl_sync(0xffffffffu, incl, 31);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {   // (a block of a grid larger than the units has no tokens: n_q = 0)
                        const int t0 = u.first + i * TPT, last = min(t0 + TPT, u.n_q) - 1;
                        const int seen = t0 >= u.n_q ? 0 : min(u.n_k, p.causal ? u.n_k - u.n_q + last + 1 : u.n_k);
                        u.tiles[i] = seen <= 0 || i >= ROW_TILES ? 0 : (seen + kKeys - 1) / kKeys;
                    }
                    u.split = ROW_TILES == 1 && u.tiles[0] > 1;
                    if (u.split) {
                        u.tiles[1] = u.tiles[0] / 2;
                        u.tiles[0] -= u.tiles[1];
                    }
                }
                if (it >= 2) ok = mbar_wait(unit_empty + 8 * (it & 1), (it >> 1) + 1 & 1, &s_abort, status, 9);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) {
                    s_unit[it & 1] = u;
                    mbar_arrive(unit_full + 8 * (it & 1));
                }
                if (block < 0) break;
                if (lane == 0) {
                    mbar_expect_tx(answered, 16);
                    take_block(smem_u32(s_answer), answered);
                    const int n_tiles = u.split ? u.tiles[0] + u.tiles[1] : max(u.tiles[0], u.tiles[1]);
                    if (n_tiles > 0) {
                        if (full_units > 0) ok = mbar_wait(q_empty, full_units + 1 & 1, &s_abort, status, 1);
                        if (ok) {
                            const int n_rows = u.tiles[1] > 0 && !u.split ? 2 : 1;   // (the second tile has keys whenever it has tokens and the first has)
                            mbar_expect_tx(q_full, n_rows * C::HALVES * 128 * TPT * p.G);
                            for (int i = 0; i < n_rows; ++i)
                                for (int h = 0; h < C::HALVES; ++h)
                                    tma_load_3d(q_smem + i * C::TILE + h * C::HALF, &tm_q, h * 64, u.group * p.G, u.q0 + u.first + i * TPT, q_full);
                        }
                        for (int c = 0; ok && c < 2 * n_tiles; ++c, ++loaded) {
                            if (loaded >= C::SLOTS) ok = mbar_wait(kv_empty + 8 * slot, loaded / C::SLOTS + 1 & 1, &s_abort, status, 1);
                            if (!ok) break;
                            mbar_expect_tx(kv_full + 8 * slot, C::TILE);
                            for (int h = 0; h < C::HALVES; ++h)
                                tma_load_3d(ring + slot * C::TILE + h * C::HALF, c & 1 ? &tm_v : &tm_k, h * 64, u.group, u.k0 + (c >> 1) * kKeys,
                                            kv_full + 8 * slot);
                            if (++slot == C::SLOTS) slot = 0;
                        }
                        ++full_units;
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ok = __all_sync(0xffffffffu, mbar_wait(answered, it & 1, &s_abort, status, 9));
                if (!ok) break;
                block = taken_block(smem_u32(s_answer));
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the next answer goes to the same place)
                __syncwarp();
            }
        } else if (warp == 9) {
            const uint32_t idesc_s = umma_idesc_bf16(128, kKeys);
            const uint32_t idesc_o = umma_idesc_bf16(128, D) | 1u << 16;   // B with N contiguous
            constexpr uint32_t kTileLow = C::TILE >> 4, kHalfLow = C::HALF >> 4;   // in units of 16 bytes
            const uint32_t q_low = desc_low(q_smem), k_low = desc_low(ring), v_low = desc_low_rows_are_k(ring);
            bool ok = true;
            int k_slot = 0, v_slot = 1, k_round = 0, v_round = 0, full_units = 0;   // ring slots of the next K and V tile, how often each went round
            int done[2] = {0, 0};                                                  // key tiles of either row tile in front of this unit
            Unit u;
            for (int it = 0; ok && next_unit(it, u); ++it) {
                // (every lane has the same; said so that the compiler can keep addresses in uniform registers)
                const int n_k = __shfl_sync(0xffffffffu, u.n_k, 0);
                const int tiles[2] = {__shfl_sync(0xffffffffu, u.tiles[0], 0), __shfl_sync(0xffffffffu, u.tiles[1], 0)};
                const bool split = ROW_TILES == 1 && __shfl_sync(0xffffffffu, u.split, 0);
                const int n = max(tiles[0], tiles[1]);
                if (n == 0) continue;
                auto wait_for = [&](uint32_t bar, int parity, uint32_t code) {
                    ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, &s_abort, status, code));
                    tc_fence_after();
                };
                auto scores = [&](int i, uint32_t a) {   // S_i = Q K^T with the Q tile at a and the K tile at k_slot
                    const uint32_t b = k_low + k_slot * kTileLow;
#pragma unroll
                    for (int s = 0; s < D / 16; ++s)
                        mma_smem(tmem + i * kKeys, a + (s >> 2) * kHalfLow + (s & 3) * 2, b + (s >> 2) * kHalfLow + (s & 3) * 2, idesc_s, s > 0);
                    umma_commit(s_full + 8 * i);
                };
                auto next_tile = [&](int &slot, int &round) {
                    slot += 2;
                    if (slot >= C::SLOTS) { slot -= C::SLOTS; ++round; }
                };
                // keys behind the sequence's last in the V tile at v_slot, which has `rows` of it: zeros
                auto clear_tail = [&](int rows) {
                    if (rows >= kKeys) return;
                    for (int e = lane; e < (kKeys - rows) * C::HALVES * 8; e += 32) {
                        const uint32_t at = ring + v_slot * C::TILE + (e / ((kKeys - rows) * 8)) * C::HALF + rows * 128 + e % ((kKeys - rows) * 8) * 16;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                };
                auto product = [&](int i, bool first) {   // O_i (+)= P_i V with the V tile at v_slot
                    const uint32_t v = v_low + v_slot * kTileLow;
#pragma unroll
                    for (int s = 0; s < kKeys / 16; ++s)
                        mma_tmem(tmem + 256 + i * 128, tmem + i * kKeys + s * 8, v + s * (2048 >> 4), idesc_o, !first || s > 0);
                    umma_commit(o_done + 8 * i);
                };
                wait_for(q_full, full_units & 1, 2);
                ++full_units;
                if (split) {   // half i has key tiles i, i + 2, ..: the ring's tiles are for one half each
                    const int all = tiles[0] + tiles[1];
                    for (int i = 0; i < 2 && ok; ++i) {
                        wait_for(kv_full + 8 * k_slot, k_round & 1, 3);
                        if (ok && elect_one()) {
                            scores(i, q_low);
                            umma_commit(kv_empty + 8 * k_slot);
                            if (i + 1 == all) umma_commit(q_empty);
                        }
                        __syncwarp();
                        next_tile(k_slot, k_round);
                    }
                    for (int kt = 0; kt < all && ok; ++kt) {
                        const int i = kt & 1, j = kt >> 1;
                        wait_for(kv_full + 8 * v_slot, v_round & 1, 3);
                        if (ok) clear_tail(n_k - kt * kKeys);
                        if (ok && kt + 2 < all) wait_for(kv_full + 8 * k_slot, k_round & 1, 3);
                        if (ok) wait_for(p_full + 8 * i, done[i] + j & 1, 4);
                        if (ok && elect_one()) {
                            product(i, j == 0);
                            umma_commit(kv_empty + 8 * v_slot);
                            if (kt + 2 < all) {
                                scores(i, q_low);
                                umma_commit(kv_empty + 8 * k_slot);
                                if (kt + 3 == all) umma_commit(q_empty);   // (the unit's last scores are issued)
                            }
                        }
                        __syncwarp();
                        next_tile(v_slot, v_round);
                        if (kt + 2 < all) next_tile(k_slot, k_round);
                    }
                    if (!ok) break;
                    done[0] += tiles[0];
                    done[1] += tiles[1];
                    continue;
                }
                if (ok) wait_for(kv_full + 8 * k_slot, k_round & 1, 3);
                if (!ok) break;
                if (elect_one()) {
                    if (tiles[0] > 0) scores(0, q_low);
                    if (tiles[1] > 0) scores(1, q_low + kTileLow);
                    umma_commit(kv_empty + 8 * k_slot);
                    if (n == 1) umma_commit(q_empty);
                }
                __syncwarp();
                next_tile(k_slot, k_round);
                for (int j = 0; j < n; ++j) {
                    wait_for(kv_full + 8 * v_slot, v_round & 1, 3);
                    if (!ok) break;
                    clear_tail(n_k - j * kKeys);
                    if (j + 1 < n) wait_for(kv_full + 8 * k_slot, k_round & 1, 3);
                    if (!ok) break;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (j < tiles[i]) {
                            if (ok) wait_for(p_full + 8 * i, done[i] + j & 1, 4);
                            if (ok && elect_one()) {
                                product(i, j == 0);
                                if (i == 1) umma_commit(kv_empty + 8 * v_slot);
                                if (j + 1 < tiles[i]) scores(i, q_low + i * kTileLow);   // over the columns that the product just issued reads
                            }
                        } else if (i == 1 && elect_one()) {
                            umma_commit(kv_empty + 8 * v_slot);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (j + 1 < n && elect_one()) {
                        umma_commit(kv_empty + 8 * k_slot);
                        if (j + 2 == n) umma_commit(q_empty);   // (the unit's last scores are issued)
                    }
                    __syncwarp();
                    next_tile(v_slot, v_round);
                    if (j + 1 < n) next_tile(k_slot, k_round);
                }
                done[0] += tiles[0];
                done[1] += tiles[1];
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int i = warp >> 2, row = tid & 127;
        const int row_token = row / p.G, row_head = row - row_token * p.G;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;          // 32 * (warp % 4) tensor-memory lanes
        const uint32_t s_at = tmem + i * kKeys + lanes, o_at = tmem + 256 + i * 128 + lanes;
        bool ok = true;
        int done = 0, met = 0;   // key tiles in front of this unit; meetings
        auto meet = [&]() {      // of both halves; bounded, as every wait
            tc_fence_before();
            mbar_arrive(met_all);
            if (ok) ok = mbar_wait(met_all, met & 1, &s_abort, status, 10);
            ok = __all_sync(0xffffffffu, ok);
            ++met;
            tc_fence_after();
        };
        Unit u;
        for (int it = 0; ok && next_unit(it, u); ++it) {
            const int n = u.tiles[i], t0 = u.first + (ROW_TILES == 1 ? 0 : i * TPT), token = t0 + row_token;
            const bool used = row_token < TPT && token < u.n_q && (ROW_TILES == 2 || i == 0 || u.split);
            const int limit = !used ? 0 : max(0, min(u.n_k, p.causal ? u.n_k - u.n_q + token + 1 : u.n_k));
            const int kt_step = ROW_TILES == 1 && u.split ? 2 : 1, kt_first = ROW_TILES == 1 && u.split ? i : 0;   // key tiles of this half
            const int all_see = min(u.n_k, p.causal ? u.n_k - u.n_q + t0 + 1 : u.n_k);   // keys that every token of the tile sees
            float ref = -1e30f;
            float2 sum = make_float2(0.f, 0.f);
            for (int j = 0; j < n; ++j) {
                ok = mbar_wait(s_full + 8 * i, done + j & 1, &s_abort, status, 5);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32_issue(s_at + c * 32, x[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_wait(x[c]);
                const int kt = kt_first + j * kt_step;
                if ((kt + 1) * kKeys > all_see) {
                    const int left = limit - kt * kKeys;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (c * 32 + e >= left) x[c][e] = 0xff800000u;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        top[c] = fmaxf(top[c], fmaxf(__uint_as_float(x[c][e]), __uint_as_float(x[c][e + 1])));
                const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.sl2;
                const bool moves = now > ref + kRise;
                if (__any_sync(0xffffffffu, moves)) {
                    const float to = moves ? now : ref, shrink = fast_exp2(ref - to);
                    ref = to;
                    sum.x *= shrink;
                    sum.y *= shrink;
                    if (j > 0) {   // O_i of the key tiles before: its last product has to be done
                        ok = mbar_wait(o_done + 8 * i, done + j - 1 & 1, &s_abort, status, 6);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        tc_fence_after();
#pragma unroll 1
                        for (int b = 0; b < D / 16; ++b) rescale16(o_at + b * 16, shrink);
                    }
                }
                const float2 scale2 = make_float2(p.sl2, p.sl2), ref2 = make_float2(-ref, -ref);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float2 y = fma2(make_float2(__uint_as_float(x[c][e]), __uint_as_float(x[c][e + 1])), scale2, ref2);
                        const float2 z = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                        sum = add2(sum, z);
                        w[e / 2] = pack_bf16(z.x, z.y);
                    }
                    tmem_st16_bits(s_at + c * 16, w);
                }
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(p_full + 8 * i);
            }
            float o_scale = 0.f;
            if (ok && n > 0) {
                ok = mbar_wait(o_done + 8 * i, done + n - 1 & 1, &s_abort, status, 7);
                ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
                const float l = sum.x + sum.y;
                o_scale = l == 0.f ? 0.f : 1.f / l;
            }
            done += n;
            if (ROW_TILES == 1 && u.split) {   // the halves' sums of a row come together; either half writes half of the channels
                // (references and sums go through the place of the second Q tile, which has none)
                float2 *const rows = reinterpret_cast<float2 *>(smem_raw + (q_smem - smem_u32(smem_raw)) + C::TILE);
                rows[i * 128 + row] = make_float2(ref, sum.x + sum.y);
                meet();
                const float2 a = rows[row], b = rows[128 + row];
                const float top = fmaxf(a.x, b.x), wa = fast_exp2(a.x - top), wb = fast_exp2(b.x - top), l = a.y * wa + b.y * wb;
                const float inv = l == 0.f ? 0.f : 1.f / l, fa = limit > 0 ? wa * inv : 0.f, fb = limit > 0 ? wb * inv : 0.f;
                char *to = p.out + (int64_t)(u.q0 + token) * p.out_token + (int64_t)(u.group * p.G + row_head) * p.out_head + i * D;
#pragma unroll 1
                for (int c = 0; c < D / 64 && ok; ++c) {
                    uint32_t oa[32], ob[32];
                    tmem_ld32_issue(tmem + 256 + lanes + i * (D / 2) + c * 32, oa);
                    tmem_ld32_issue(tmem + 384 + lanes + i * (D / 2) + c * 32, ob);
                    tmem_ld_wait(oa);
                    tmem_ld_wait(ob);
                    if (used) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t w[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                const int k = 8 * e + 2 * x;
                                w[x] = limit > 0 ? pack_bf16(fmaf(__uint_as_float(oa[k]), fa, __uint_as_float(ob[k]) * fb),
                                                             fmaf(__uint_as_float(oa[k + 1]), fa, __uint_as_float(ob[k + 1]) * fb)) : 0;
                            }
                            *reinterpret_cast<uint4 *>(to + c * 64 + e * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                }
                meet();   // (the next unit's products go over both halves' sums)
                continue;
            }
            if (ok) {
                char *to = p.out + (int64_t)(u.q0 + token) * p.out_token + (int64_t)(u.group * p.G + row_head) * p.out_head;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    if (n > 0) {
                        tmem_ld32_issue(o_at + c * 32, o);
                        tmem_ld_wait(o);
                    }
                    if (used) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t w[4];
#pragma unroll
                            for (int b = 0; b < 4; ++b)
                                w[b] = n > 0 && limit > 0 ? pack_bf16(__uint_as_float(o[8 * e + 2 * b]) * o_scale, __uint_as_float(o[8 * e + 2 * b + 1]) * o_scale) : 0;
                            *reinterpret_cast<uint4 *>(to + c * 64 + e * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                }
            }
        }
    }
    // Every copy and product has been waited for by the roles above unless a wait gave up; then the ones in flight get
    // their time (bounded) before the block's memory goes.
    tc_fence_before();
    __syncthreads();
    if (s_abort && tid == 0) {
        atomicAdd(&g_prompt_timeouts, 1);
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
}

// bf16 rows of heads as a 3-D tensor (d, heads, tokens); a box is 64 channels x `heads` x `tokens`.
int tokens_map(CUtensorMap *tm, const aircache_tokens_t *t, int d, int heads, int64_t tokens, int box_heads, int box_tokens) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) { set_last_cuda_error(cudaErrorSymbolNotFound); return AIRCACHE_ERR_CUDA; }
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)(heads > 1 ? t->stride_head * 2 : d * 2),
                                   (cuuint64_t)(tokens > 1 ? t->stride_token * 2 : d * 2)};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens}, estr[3] = {1, 1, 1};
    const CUresult rc = fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, t->data, dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? AIRCACHE_OK : AIRCACHE_ERR_UNSUPPORTED;
}

template <int D, int ROW_TILES>
int launch_d(const CUtensorMap &tm_q, const CUtensorMap &tm_k, const CUtensorMap &tm_v, const PromptParams &p, int dev, cudaStream_t st) {
    static std::atomic<uint64_t> allowed[kMaxDevices];
    const int rc = allow_shared_memory((const void *)prompt_kernel<D, ROW_TILES>, PromptCfg<D>::SMEM, dev, allowed);
    if (rc) return rc;
    return launch_dependent(prompt_kernel<D, ROW_TILES>, dim3((unsigned)(p.units * p.n_kv_heads)), dim3(PromptCfg<D>::THREADS), PromptCfg<D>::SMEM, st,
                            tm_q, tm_k, tm_v, p);
}

}  // namespace

int launch_prompt(const aircache_prompt_t *s, const aircache_tokens_t *q, const aircache_tokens_t *k,
                  const aircache_tokens_t *v, const int32_t *q_offsets, const int32_t *k_offsets,
                  const aircache_tokens_t *out, cudaStream_t st) {
    PromptParams p = {};
    p.q_offsets = q_offsets;
    p.k_offsets = k_offsets ? k_offsets : q_offsets;
    p.out = static_cast<char *>(out->data);
    p.out_token = 2 * out->stride_token;
    p.out_head = 2 * out->stride_head;
    p.n_seqs = s->n_seqs;
    p.q_tokens = s->q_tokens;
    p.k_tokens = s->k_tokens;
    p.n_kv_heads = s->n_kv_heads;
    p.G = s->n_q_heads / s->n_kv_heads;
    p.tokens_per_tile = 128 / p.G;
    int dev = 0, sms = 0, rc = current_device(&dev, &sms);
    if (rc) return rc;
    p.causal = s->causal;
    p.sl2 = s->scale * kLog2e;
    // One row tile a block, its keys shared by the block's halves, where every block then has an SM of its own: 640 tokens of
    // a small model 14.0 -> 10.3 us.  In calls of more blocks it reads the keys twice as often (16 turns of 1 to 202 tokens
    // over some 2000 keys each, 116 blocks of two row tiles: 52 us, 65 with one a block).  The count is the host's bound on blocks, a
    // tile a sequence too many; where most sequences are a token or two, second row tiles are empty (not measured apart).
    const int row_tiles = ((int64_t)s->q_tokens / p.tokens_per_tile + s->n_seqs) * s->n_kv_heads <= sms ? 1 : 2;
    const int64_t units = s->q_tokens / (row_tiles * p.tokens_per_tile) + s->n_seqs;   // at least as many as there are
    if (units * s->n_kv_heads >= ((int64_t)1 << 31)) return AIRCACHE_ERR_UNSUPPORTED;
    p.units = (int)units;
    CUtensorMap tm_q, tm_k, tm_v;
    if ((rc = tokens_map(&tm_q, q, s->head_dim, s->n_q_heads, s->q_tokens, p.G, p.tokens_per_tile))) return rc;
    const bool keys = s->k_tokens > 0;   // (without keys nothing is loaded)
    if ((rc = tokens_map(&tm_k, keys ? k : q, s->head_dim, keys ? s->n_kv_heads : 1, keys ? s->k_tokens : 1, 1, kKeys))) return rc;
    if ((rc = tokens_map(&tm_v, keys ? v : q, s->head_dim, keys ? s->n_kv_heads : 1, keys ? s->k_tokens : 1, 1, kKeys))) return rc;
    if (row_tiles == 1)
        return s->head_dim == 64 ? launch_d<64, 1>(tm_q, tm_k, tm_v, p, dev, st) : launch_d<128, 1>(tm_q, tm_k, tm_v, p, dev, st);
    return s->head_dim == 64 ? launch_d<64, 2>(tm_q, tm_k, tm_v, p, dev, st) : launch_d<128, 2>(tm_q, tm_k, tm_v, p, dev, st);
}

// The count on the device only grows.  What a stream has seen of it is kept here, under the ids of its context and its own (a
// handle may come again): no check takes a failure from another one, and none can get lost between a read and a reset.
// (More streams than places: the oldest is forgotten, and would be told of a failure a second time.)
struct Seen { uint64_t context; unsigned long long stream; uint32_t count; };

int prompt_status(cudaStream_t st) {
    static std::mutex lock;
    static Seen seen[256];
    static int n = 0, oldest = 0;
    uint32_t count = 0;
    unsigned long long id = 0;
    AIRCACHE_CUDA_TRY(cudaStreamGetId(st, &id));
    AIRCACHE_CUDA_TRY(cudaMemcpyFromSymbolAsync(&count, g_prompt_timeouts, sizeof count, 0, cudaMemcpyDeviceToHost, st));
    AIRCACHE_CUDA_TRY(cudaStreamSynchronize(st));
    const uint64_t context = context_id();
    const std::lock_guard<std::mutex> hold(lock);
    int at = 0;
    while (at < n && (seen[at].context != context || seen[at].stream != id)) ++at;
    if (at == n) {
        if (count == 0) return AIRCACHE_OK;
        if (n < 256) {
            ++n;
        } else {
            at = oldest;
            oldest = (oldest + 1) % 256;
        }
        seen[at] = {context, id, 0};
    }
    const bool more = (int32_t)(count - seen[at].count) > 0;   // (not behind what another thread's check of this stream has read)
    if (more) seen[at].count = count;
    return more ? AIRCACHE_ERR_TIMEOUT : AIRCACHE_OK;
}

// A wait that nobody ends, counted as one of prompt_kernel's.
namespace {
__global__ void prompt_timeout_kernel() {
    __shared__ uint64_t s_bar;
    __shared__ volatile int s_abort;
    __shared__ uint32_t s_status;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&s_bar), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_abort = 0;
    }
    __syncthreads();
    mbar_wait(smem_u32(&s_bar), 0, &s_abort, &s_status, 11);
    __syncthreads();
    if (s_abort && threadIdx.x == 0) atomicAdd(&g_prompt_timeouts, 1);
}
}  // namespace

int launch_prompt_timeout(cudaStream_t st) {
    prompt_timeout_kernel<<<1, 64, 0, st>>>();
    AIRCACHE_LAUNCH_CHECK();
    return AIRCACHE_OK;
}

}  // namespace aircache
