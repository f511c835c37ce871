// Attention of chunks of new tokens over the paged cache on the tensor cores (tcgen05).
//
// A CTA works on row tiles of 128 packed rows (row = token * G + head) against blocks of keys:
//     S = Q K^T        tcgen05.mma, operands in shared memory, S (fp32) in tensor memory
//     P = 2^(c S - m)  running maximum m and sum l per row; P (bf16) in tensor memory, two buffers per tile
//     O += P V         A = P from tensor memory, B = V as it lies (rows are the contraction index: MN-major)
// head_dim <= 128: two row tiles against blocks of 64 keys (S, P and O of both fill the 512 columns of tensor memory).
// head_dim 256: O of one tile takes half of them, so there is one tile, against blocks of 128 keys, and two CTAs of a
// cluster work as one (cta_group::2): 256 rows, each CTA with its 128, half of a block's keys of K and half of V's
// channels.  What an SM can draw from L2 (26 to 29 bytes per cycle) was the limit of a CTA alone, which fetches 64 KiB of K and
// V for 128 rows and 64 keys; a CTA of the pair fetches half of that (512 tokens over 16 384 keys, 8 lists: 206 -> 122 us, the
// tensor pipe 67 % busy).  The last row tile of a list costs as much as a full one: 517 tokens take 148 us where 512 take 125.
//
// Two warps keep K and V flowing through a ring of slots each (TMA boxes of a page), one warp per row tile issues its MMAs
// (the waits of one are hidden by the other's; in a pair one warp of the first CTA issues for both), eight warps do the
// softmax, 64 scores per thread and block.  The scores of the next block are on their way as soon as those of this one
// have been read.  A row tile of at most 128 rows leaves the second place of a CTA free at head_dim <= 128: both take
// every other block of it, and the first takes the second's output in at the end (128 lists of 8192 keys, 20 to 32 rows:
// head_dim 64 102 -> 74 us, 128 123 -> 115).
//
// The running maximum only moves when a row's scores exceed it by more than 2^8 (the weights then stay within fp32 and
// bf16 range, and the sum, which uses the same maximum, cancels it): O is rescaled in tensor memory only then.
//
// The CTAs divide the call's (row tile, key block) units evenly, as in the kernel for few rows (paged_attn.cuh).
//
// What bounds it at head_dim 128: for 64 keys and two tiles the MMAs take 1280 cycles (Q K^T with N = 64 reads its 128
// query rows from shared memory for only 64 columns: 48 cycles an instruction where the arithmetic takes 32), the
// exponentials 1024 of the special function units; the two tiles alternate on both and about 1600 pass.  2048 tokens
// over 32 768 keys, 32 heads on 8 lists: 880 us = 1.21 PFLOP/s (0.72 of the measured cuBLAS rate); back to back, at the
// clock that the power limit leaves, 1040 to 1080 us (0.70 to 0.73 of the rate measured there).  At head_dim 64 the exponentials
// are the larger part: 1024 tokens over 16 384 keys take 194 us, the special function units 68 % busy, the tensor pipe 34 %.
#include <type_traits>

#include "paged.h"
#include "paged_attn.cuh"
#include "ptx_sm100.cuh"

using namespace ptx;

namespace {

constexpr float kRescale = 8.0f;          // log2 of how far a row's scores may exceed its running maximum

template <int D> struct Chunk {
    static constexpr bool PAIR = D == 256;              // two CTAs of a cluster work as one
    static constexpr int TILES = PAIR ? 1 : 2;          // row tiles of a CTA
    static constexpr int HALVES = 2 / TILES;            // threads per row (each has 64 keys of a block)
    static constexpr int ROWS = 256;
    static constexpr int BK = HALVES * 64;              // keys per block
    // a slot of its ring: K: KROWS keys x KW * 64 channels;  V: VKEYS keys x VCH channels (a CTA of a pair: half the keys of
    // a block for K, half the channels for V)
    static constexpr uint32_t SLOT = D == 64 ? 8192 : 16384;
    static constexpr int KROWS = PAIR ? BK / 2 : BK, KW = (int)SLOT / (KROWS * 128), KC = D / 64 / KW;
    static constexpr int VCH = PAIR ? D / 2 : D, VKEYS = (int)SLOT / (VCH * 2), VC = BK / VKEYS;
    static constexpr uint32_t Q_TILE = 128u * D * 2;
    static constexpr int NSLOT = D == 64 ? 20 : D == 128 ? 10 : 9, NV = NSLOT / 2, NK = NSLOT - NV;   // K's ring, then V's
    static constexpr int PARTS = PAIR ? kPagedMaxCtas : 2 * kPagedMaxCtas;             // places for parts of a row tile
    static constexpr int THREADS = 128 + 256;           // warps 0 and 3 (K, V), 1 and 2 (MMA of a row tile), then the softmax warps
    static constexpr int BARS = 2 * NSLOT + 18;
    static constexpr int TAIL_WALK = (BARS * 8 + 16 + 7) / 8 * 8;
    static constexpr int TAIL_STATS = TAIL_WALK + (int)sizeof(Walk);
    // two threads per row: [turn][half][row] maxima; two tiles: [row] maxima and sums of a split item
    static constexpr int TAIL = TAIL_STATS + (HALVES == 2 ? 2 * 2 * 128 * 4 : 128 * 8);
    static constexpr int SMEM = 1024 + (int)(TILES * Q_TILE) + NSLOT * (int)SLOT + TAIL;
    static constexpr uint32_t O_COL = 256;              // tensor memory: S of tile t at 2 t BK, P of buffer b BK + b BK / 2 on, O from 256
    static_assert(SMEM + 256 <= 232448, "a CTA's shared memory, with room for static arrays");
    static_assert(KC * KW * 64 == D && VC * VKEYS == BK && VKEYS % 16 == 0 && NV >= VC && NK >= KC && (!PAIR || NV < 3 * VC), "slots");
};

// A place in the ring: slot, and the parity of its use.
struct Ring {
    uint32_t slot, phase;
    __device__ __forceinline__ void next(int first, int end) {
        if (++slot == (uint32_t)end) {
            slot = (uint32_t)first;
            phase ^= 1;
        }
    }
};

template <int D>
__global__ void __launch_bounds__(Chunk<D>::THREADS, 1)
paged_chunk_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const AttnArgs a) {
    using C = Chunk<D>;
    constexpr int NS = C::NSLOT, BK = C::BK;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t s_q = base, s_ring = base + C::TILES * C::Q_TILE;
    const uint32_t bars = s_ring + NS * C::SLOT;
    uint8_t* tail = gen + C::TILES * C::Q_TILE + NS * C::SLOT;
    auto full = [&](uint32_t s) { return bars + 8u * s; };
    auto empty = [&](uint32_t s) { return bars + 8u * (NS + s); };
    // per row tile t (and buffer b of the weights): scores written, scores read, weights written, product done
    auto s_full = [&](int t) { return bars + 8u * (2 * NS + t); };
    auto s_read = [&](int t) { return bars + 8u * (2 * NS + 2 + t); };
    auto p_full = [&](int t, int b) { return bars + 8u * (2 * NS + 4 + 2 * t + b); };
    auto o_done = [&](int t, int b) { return bars + 8u * (2 * NS + 8 + 2 * t + b); };
    auto q_full = [&](int t) { return bars + 8u * (2 * NS + 12 + t); };
    auto drained = [&](int t) { return bars + 8u * (2 * NS + 14 + t); };      // only used when a wait has given up
    // (pair) V of the blocks that reach behind their list, on this CTA's own barriers, in turn: V's ring holds two blocks
    auto v_tail = [&](uint32_t use) { return bars + 8u * (2 * NS + 16 + (use & 1)); };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail + 8 * C::BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8 * C::BARS + 4);
    volatile int* last_flag = abort_flag + 1;           // per row tile: this CTA joins its parts
    Walk* start = reinterpret_cast<Walk*>(tail + C::TAIL_WALK);

    // in a pair: this CTA's place, and what stands for a CTA elsewhere
    const int rank = C::PAIR ? (int)cluster_ctarank() : 0;
    const int worker = C::PAIR ? (int)blockIdx.x / 2 : (int)blockIdx.x, workers = C::PAIR ? (int)gridDim.x / 2 : (int)gridDim.x;
    // an arrival on the MMA issuer's barrier
    auto tell = [&](uint32_t bar) {
        if (C::PAIR) mbar_arrive_cluster(mapa(bar, 0));
        else mbar_arrive(bar);
    };
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), C::TILES);
        }
        for (int t = 0; t < 2; ++t) {
            for (int b = 0; b < 2; ++b) {
                mbar_init(p_full(t, b), C::PAIR ? 16 : 4);
                mbar_init(o_done(t, b), 1);
            }
            mbar_init(s_full(t), 1);
            mbar_init(s_read(t), C::PAIR ? 16 : 4);
            mbar_init(q_full(t), C::PAIR ? 16 : 4);
            mbar_init(drained(t), 1);
        }
        for (int i = 0; i < 2; ++i) mbar_init(v_tail(i), C::VC);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&k_map);
        prefetch_tensormap(&v_map);
    }
    if (warp == 1) {
        if (C::PAIR) {
            tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
            tmem_relinquish();
        }
    }
    find_range<C::THREADS>(a, BK, C::ROWS, worker, workers, start);
    tc_fence_before_sync();
    __syncthreads();
    if (C::PAIR) cluster_sync();                        // the peer's barriers exist before anything signals them
    tc_fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    Walk walk = *start;
    Item it;
    bool ok = true;

    // ---------------------------------------------------------------------------------- K (warp 0) or V (warp 3)
    auto feed = [&](auto is_v) {
        constexpr bool V = decltype(is_v)::value;
        // a slot: ROWS keys and WIDE times 64 channels; CHUNKS of them a block
        constexpr int ROWS = V ? C::VKEYS : C::KROWS, WIDE = V ? C::VCH / 64 : C::KW, CHUNKS = V ? C::VC : C::KC;
        constexpr int FIRST = V ? C::NK : 0, END = V ? NS : C::NK, MAX_SHIFT = ROWS == 128 ? 7 : ROWS == 64 ? 6 : 5;
        const uint32_t leader = elect_one();
        const int box_shift = min(a.shift, MAX_SHIFT), row_mask = (1 << a.shift) - 1;      // keys of a box
        Ring ring = {FIRST, 0};
        uint32_t tails = 0;
        while (next_item(a, walk, C::ROWS, BK, it)) {
            const int n = it.li.n;
            const int entries = (int)(((unsigned)n + (1u << a.shift) - 1u) >> a.shift);
            const int32_t* tab = a.table + (size_t)it.list * a.max_pages;
            auto entry = [&](int e) {
                int page = 0;
                if (e < entries) {
                    page = tab[e];
                    if ((unsigned)page >= (unsigned)a.n_pages) {
                        a.status[1] = (int)EA_ERR_PAGES;
                        page = 0;
                    }
                }
                return page;
            };
            // table entries ride in registers, 32 ahead of the 32 in use
            int win = (int)(((long long)it.b0 * BK) >> a.shift) & ~31;
            int cur = entry(win + lane), next = entry(win + 32 + lane);
            for (int b = it.b0; b < it.b1; ++b) {
                if (((b * BK) >> a.shift) >= win + 32) {
                    win += 32;
                    cur = next;
                    next = entry(win + 32 + lane);
                }
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    const int key0 = b * BK + (V ? c * ROWS : rank * ROWS), rest = n - key0;
                    auto boxes_of = [&](int left) { return left <= 0 ? 0 : min(ROWS >> box_shift, (left + (1 << box_shift) - 1) >> box_shift); };
                    const int boxes = boxes_of(rest);
                    if (ok) ok = mbar_wait(empty(ring.slot), ring.phase ^ 1, abort_flag);
                    __syncwarp();
                    const uint32_t go = ok ? leader : 0u;
                    const uint32_t to = s_ring + ring.slot * C::SLOT;
                    uint32_t bar = full(ring.slot);
                    // V rows behind the list's end are made zero by the softmax warps, which in a pair can only wait for this
                    // CTA's part of the block: it gets a barrier of its own, and the weights' arrival tells the MMA issuer
                    const bool own = C::PAIR && V && (b + 1) * BK > n;
                    if (!C::PAIR) {
                        if (go) mbar_arrive_expect_tx(bar, (uint32_t)((boxes * 128 * WIDE) << box_shift));
                    } else {
                        // in a pair the leader's barrier counts both CTAs' bytes: V alike, K the two halves of the keys
                        const int both = own ? 0 : V ? 2 * boxes : boxes + boxes_of(rest - ROWS);
                        if (go && rank == 0) mbar_arrive_expect_tx(bar, (uint32_t)((both * 128 * WIDE) << box_shift));
                        if (go && own) mbar_arrive_expect_tx(v_tail(tails), (uint32_t)((boxes * 128 * WIDE) << box_shift));
                        bar = own ? v_tail(tails) : mapa(bar, 0);
                    }
                    auto load = [&](uint32_t dst, const CUtensorMap* map, int y, int z) {
                        if (C::PAIR && !own) tma_load_3d_pair_warp(go, dst, map, bar, 0, y, z);
                        else tma_load_3d_warp(go, dst, map, bar, 0, y, z);
                    };
#pragma unroll 2
                    for (int x = 0; x < boxes; ++x) {
                        const int key = key0 + (x << box_shift);
                        const int y = (__shfl_sync(0xffffffffu, cur, ((key >> a.shift) - win) & 31) << a.shift) + (key & row_mask);
                        if (V) {                        // box after box: [64 channels][row][128 bytes] each
                            load(to + ((uint32_t)(x * C::VCH * 2) << box_shift), &v_map, y, rank * WIDE);
                        } else {                        // the rows of a chunk of 64 channels side by side
#pragma unroll
                            for (int w = 0; w < WIDE; ++w) load(to + w * ROWS * 128 + ((uint32_t)(x * 128) << box_shift), &k_map, y, c * WIDE + w);
                        }
                    }
                    ring.next(FIRST, END);
                }
                if ((b + 1) * BK > n) ++tails;
            }
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok && lane == 0)
            for (int s = FIRST; s < END; ++s) {         // copies in flight land before the shared memory goes away
                mbar_drain(full(s), 0);
                mbar_drain(full(s), 1);
            }
        if (C::PAIR && V && !ok && lane == 0)
            for (int i = 0; i < 4; ++i) mbar_drain(v_tail(i), i / 2);
        __syncwarp();
    };
    if (warp == 0) {
        feed(std::false_type());
    } else if (warp == 3) {
        feed(std::true_type());
    } else if (warp <= C::TILES && rank == 0) {
        // ------------------------------------------------------------------------------ MMA issuer of a row tile
        // The whole warp runs this loop in step, and one lane issues (see umma_bf16_warp).
        const int t = warp - 1;
        const uint32_t leader = elect_one();
        const uint32_t idesc_s = C::PAIR ? umma_idesc_bf16_m256(BK) : umma_idesc_bf16_m128(BK);
        const uint32_t idesc_o = (C::PAIR ? umma_idesc_bf16_m256(D) : umma_idesc_bf16_m128(D)) | kIdescBMnMajor;
        auto commit = [&](uint32_t bar) {               // (in a pair: on both CTAs' barriers)
            if (C::PAIR) umma_commit_pair_warp(leader, bar, 3);
            else umma_commit_warp(leader, bar);
        };
        const uint64_t q_desc = umma_desc_k_sw128(s_q + t * C::Q_TILE), k_desc = umma_desc_k_sw128(s_ring);
        // V: a box of `vbox` keys after the other, in it a chunk of 64 channels after the other
        const int vbox = min(1 << a.shift, C::VKEYS), vbits = vbox == C::VKEYS ? 31 : a.shift;
        const uint64_t v_desc = umma_desc_mn_sw128(s_ring, (uint32_t)vbox * 128u);
        uint64_t v_step[C::VKEYS / 16];                 // to keys 16 ks ..: box (16 ks) / vbox, row (16 ks) % vbox of it
#pragma unroll
        for (int ks = 0; ks < C::VKEYS / 16; ++ks)
            v_step[ks] = (uint32_t)__shfl_sync(0xffffffffu, ((ks * 16 >> vbits) * vbox * (C::VCH * 2 - 128) + ks * 2048) >> 4, 0);
        const uint32_t s_tmem = tmem + 2 * t * BK, o_tmem = tmem + C::O_COL + t * D;
        uint32_t p_phase = 0, q_phase = 0, r_phase = 0; // parity of the next phase of p_full(t, b) (bit b), q_full, s_read
        Ring k_ring = {0, 0}, v_ring = {(uint32_t)C::NK, 0};
        while (next_item(a, walk, C::ROWS, BK, it)) {
            const int count = __shfl_sync(0xffffffffu, it.b1 - it.b0, 0);
            const bool split = __shfl_sync(0xffffffffu, C::TILES == 2 && it.li.rows_tok * a.G - it.tile * C::ROWS <= 128, 0);
            const int mine = split ? (count + 1 - t) / 2 : count;      // blocks t, t + 2, .. or all of them
            // blocks that the other warp works on: their slots are only given back
            auto skip = [&](Ring& ring, int slots, int first, int end) {
#pragma unroll 1
                for (int c = 0; c < slots; ++c) {
                    if (ok) ok = mbar_wait<C::PAIR>(full(ring.slot), ring.phase, abort_flag);
                    if (leader) mbar_arrive(empty(ring.slot));
                    ring.next(first, end);
                }
            };
            // (two copies: what a split item adds would cost the others a few percent)
            auto work = [&](auto is_split) {
                constexpr bool SPLIT = decltype(is_split)::value;
                if (SPLIT && mine == 0) {
                    skip(k_ring, C::KC, 0, C::NK);
                    skip(v_ring, C::VC, C::NK, NS);
                    return;
                }
                if (ok) ok = mbar_wait<C::PAIR>(q_full(t), q_phase, abort_flag);
                q_phase ^= 1;
#pragma unroll 1
                for (int j = -1; j < mine; ++j) {
                    if (j + 1 < mine) {                     // S = Q K(j + 1)^T, once the softmax has read the scores before
                        if (SPLIT) skip(k_ring, (j < 0 ? t : 1) * C::KC, 0, C::NK);
                        if (j >= 0) {
                            if (ok) ok = mbar_wait<C::PAIR>(s_read(t), r_phase, abort_flag);
                            r_phase ^= 1;
                        }
#pragma unroll
                        for (int c = 0; c < C::KC; ++c) {
                            if (ok) ok = mbar_wait<C::PAIR>(full(k_ring.slot), k_ring.phase, abort_flag);
                            ok = __all_sync(0xffffffffu, ok);
                            if (ok) {
                                tc_fence_after_sync();
                                const uint64_t qd = q_desc + c * C::KW * (16384 >> 4), kd = k_desc + k_ring.slot * (C::SLOT >> 4);
#pragma unroll
                                for (int ks = 0; ks < 4 * C::KW; ++ks) {
                                    const uint64_t q_at = qd + (ks / 4) * (16384 >> 4) + ks % 4 * 2;
                                    const uint64_t k_at = kd + (ks / 4) * (C::KROWS * 128 >> 4) + ks % 4 * 2;
                                    if (C::PAIR) umma_bf16_pair_warp(leader, s_tmem, q_at, k_at, idesc_s, c + ks > 0 ? 1u : 0u);
                                    else umma_bf16_warp(leader, s_tmem, q_at, k_at, idesc_s, c + ks > 0 ? 1u : 0u);
                                }
                                commit(empty(k_ring.slot));
                            }
                            k_ring.next(0, C::NK);
                        }
                        if (ok) commit(s_full(t));
                    }
                    if (j >= 0) {                           // O += P(j) V(j)
                        const int b = j & 1;
                        if (SPLIT) skip(v_ring, (j == 0 ? t : 1) * C::VC, C::NK, NS);
                        if (ok) ok = mbar_wait<C::PAIR>(p_full(t, b), (p_phase >> b) & 1, abort_flag);
                        p_phase ^= 1u << b;
#pragma unroll
                        for (int c = 0; c < C::VC; ++c) {
                            if (ok) ok = mbar_wait<C::PAIR>(full(v_ring.slot), v_ring.phase, abort_flag);
                            ok = __all_sync(0xffffffffu, ok);
                            if (ok) {
                                tc_fence_after_sync();
                                const uint64_t vd = v_desc + v_ring.slot * (C::SLOT >> 4);
                                const uint32_t p_tmem = s_tmem + BK + b * (BK / 2) + c * (C::VKEYS / 2);
#pragma unroll
                                for (int ks = 0; ks < C::VKEYS / 16; ++ks) {
                                    const uint32_t onto = c + ks > 0 ? 1u : (uint32_t)j;
                                    if (C::PAIR) umma_bf16_ts_pair_warp(leader, o_tmem, p_tmem + ks * 8, vd + v_step[ks], idesc_o, onto);
                                    else umma_bf16_ts_warp(leader, o_tmem, p_tmem + ks * 8, vd + v_step[ks], idesc_o, onto);
                                }
                                commit(empty(v_ring.slot));
                            }
                            v_ring.next(C::NK, NS);
                        }
                        if (ok) commit(o_done(t, b));
                    }
                }
                if (SPLIT && t + 2 * mine - 1 < count) {
                    skip(k_ring, C::KC, 0, C::NK);
                    skip(v_ring, C::VC, C::NK, NS);
                }
            };
            if (C::TILES == 2 && split) work(std::true_type());
            else work(std::false_type());
            ok = __all_sync(0xffffffffu, ok);
        }
        if (!ok) {                                      // MMAs in flight end before the tensor memory goes back
            commit(drained(t));
            mbar_drain(drained(t), 0);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------------------------------ softmax
        // With two row tiles four warps have one each, a thread per row; with one, warps w and w + 4 share its rows, one
        // taking keys 0-63 of a block, the other 64-127, and agree on the maximum through shared memory.
        const int t = C::TILES == 2 ? (warp - 4) / 4 : 0, half = C::HALVES == 2 ? (warp - 4) / 4 : 0, quarter = warp & 3;
        constexpr int TILE_THREADS = 128 * C::HALVES;
        const int row = quarter * 32 + lane;            // tensor-memory lanes follow warp % 4
        const int tid = threadIdx.x - 128 - t * 128;    // among the tile's threads
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        constexpr int OWN = D / C::HALVES;              // output channels of a thread
        const uint32_t o_col = tmem + lanes + C::O_COL + t * D + half * OWN;
        float* stats = reinterpret_cast<float*>(tail + C::TAIL_STATS);
        const int vbox = min(1 << a.shift, C::VKEYS);   // keys of a V box
        uint32_t s_phase = 0, turn = 0, tails = 0, uses[2] = {0, 0};   // uses: of the weights' buffers, before this item
        long long seq = 0;                              // V slots of the items before this one
        // the queries take the sign (exact), so that max(c S) = c max(S); a scale of zero becomes one that leaves nothing of
        // any score but does not make NaN of a masked one (-infinity)
        const float scale = a.scale_log2 == 0.f ? 1e-37f : fabsf(a.scale_log2);
        // the partner's value of a pair of threads (both call it, `turn` alternates the buffers)
        auto partner = [&](float mine) {
            float* at = stats + (turn & 1) * 256;
            at[half * 128 + row] = mine;
            bar_sync(1 + quarter, 64);
            ++turn;
            return at[(half ^ 1) * 128 + row];
        };
        while (next_item(a, walk, C::ROWS, BK, it)) {
            const ListInfo& li = it.li;
            const int count = it.b1 - it.b0;
            const int live_rows = li.rows_tok * a.G - it.tile * C::ROWS;
            // Two row tiles and rows for one: they split the blocks, each with its own running maximum, sum and output.
            const bool split = C::TILES == 2 && live_rows <= 128;
            const int mine = split ? (count + 1 - t) / 2 : count;
            const int part_tile = C::PAIR ? rank : split ? 0 : t;      // which 128 of a row tile's rows
            if (mine == 0) {
                seq += (long long)count * C::VC;
                continue;
            }
            // ---- queries: 16 bytes per thread and step, rows without a query are zero
            const int head0 = (it.list - quotient(it.list, a.div_hkv) * a.Hkv) * a.G;
            const int row0 = it.tile * C::ROWS + part_tile * 128;
            constexpr int PIECES = D / 8, STEPS = 128 * PIECES / TILE_THREADS, BATCH = STEPS < 8 ? STEPS : 8;
            // (the same thread that stored an output piece in this place, so the place is free)
            const uint32_t q_tile = s_q + t * C::Q_TILE;
            auto q_place = [&](int r, int piece) { return q_tile + (piece / 8) * 16384u + r * 128u + (((piece % 8) * 16u) ^ ((r & 7) * 16u)); };
#pragma unroll
            for (int i0 = 0; i0 < STEPS; i0 += BATCH) {
                uint4 v[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int at = (i0 + i) * TILE_THREADS + tid, r = at / PIECES, piece = at % PIECES;
                    const int tok = quotient(row0 + r, a.div_g), h = head0 + row0 + r - tok * a.G;
                    v[i] = make_uint4(0, 0, 0, 0);
                    if (tok < li.rows_tok)
                        v[i] = __ldg(reinterpret_cast<const uint4*>(a.q + (li.q0 + tok) * a.q_stride + (long long)h * D + piece * 8));
                }
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int at = (i0 + i) * TILE_THREADS + tid;
                    if (a.scale_log2 < 0.f) {
                        v[i].x ^= 0x80008000u;
                        v[i].y ^= 0x80008000u;
                        v[i].z ^= 0x80008000u;
                        v[i].w ^= 0x80008000u;
                    }
                    sts128(q_place(at / PIECES, at % PIECES), v[i]);
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) tell(q_full(t));

            const int tok = quotient(row0 + row, a.div_g);
            const bool live = tok < li.rows_tok;
            const int lim = live ? limit_of(li, a, tok) : 0;
            // keys that every row of the tile sees
            const int seen = limit_of(li, a, min(quotient(row0, a.div_g), li.rows_tok - 1));
            float m = -INFINITY, l = 0.f;
            // the product of block j has ended
            auto wait_product = [&](int j) {
                if (ok) ok = mbar_wait(o_done(t, j & 1), (uses[j & 1] + (uint32_t)(j >> 1)) & 1, abort_flag);
                __syncwarp();
            };
            auto softmax = [&](auto is_split) {
                constexpr bool SPLIT = decltype(is_split)::value;
#pragma unroll 1
                for (int j = 0; j < mine; ++j) {
                    const int block = SPLIT ? 2 * j + t : j, key0 = (it.b0 + block) * BK, b = j & 1;
                    if (ok) ok = mbar_wait(s_full(t), s_phase, abort_flag);
                    s_phase ^= 1;
                    if (key0 + BK > li.n) {
                        // value rows behind the list's end hold anything, and a weight of zero does not silence a NaN: they become
                        // zero before the weights let the product go (by both tiles: the zeros are the same).  (A parity tells two
                        // neighbouring phases apart: the slots' earlier use is known to be over when the product before is.)
                        if (C::PAIR) {
                            if (ok) ok = mbar_wait(v_tail(tails), (tails >> 1) & 1, abort_flag);
                            ++tails;
                        } else if (j > 0) {
                            wait_product(j - 1);
                        }
                        for (int c = 0; c < C::VC; ++c) {
                            const long long at = seq + block * C::VC + c;
                            const uint32_t s = C::NK + (uint32_t)(at % C::NV);
                            const int from = max(0, li.n - key0 - c * C::VKEYS);
                            if (from >= C::VKEYS) continue;
                            if (!C::PAIR && ok) ok = mbar_wait(full(s), (uint32_t)(at / C::NV) & 1, abort_flag);
                            constexpr int V_PIECES = C::VCH / 8;
                            for (int i = tid; i < (C::VKEYS - from) * V_PIECES; i += TILE_THREADS) {
                                const int r = from + i / V_PIECES, piece = i % V_PIECES;
                                const uint32_t box = s_ring + s * C::SLOT + (r / vbox) * vbox * (C::VCH * 2);
                                sts128(box + ((piece / 8) * vbox + r % vbox) * 128u + (piece % 8) * 16u, make_uint4(0, 0, 0, 0));
                            }
                        }
                        fence_proxy_async_smem();
                    }
                    __syncwarp();
                    tc_fence_after_sync();
                    const uint32_t s_col = tmem + lanes + 2 * t * BK;
                    uint32_t x[2][32];
                    tmem_ld_x32(s_col + half * 64, x[0]);
                    tmem_ld_x32(s_col + half * 64 + 32, x[1]);
                    tmem_ld_wait();                         // (of the whole warp)
                    tc_fence_before_sync();
                    if (lane == 0 && j + 1 < mine) tell(s_read(t));
                    if (key0 + BK > seen) {
                        const int local = lim - key0 - half * 64;
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            if (i >= local) x[i / 32][i % 32] = 0xff800000u;
                    }
                    float top[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        top[i] = __uint_as_float(x[i / 2][i % 2 * 16]);
#pragma unroll
                        for (int e = 1; e < 15; e += 2)
                            top[i] = max3(top[i], __uint_as_float(x[i / 2][i % 2 * 16 + e]), __uint_as_float(x[i / 2][i % 2 * 16 + e + 1]));
                        top[i] = fmaxf(top[i], __uint_as_float(x[i / 2][i % 2 * 16 + 15]));
                    }
                    float raw = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                    if (C::HALVES == 2) raw = fmaxf(raw, partner(raw));
                    const float m_blk = raw * scale;
                    const bool move = m_blk > m + kRescale; // (a row that has seen nothing has m = -infinity)
                    if (__any_sync(0xffffffffu, move)) {
                        // (below the range the maximum stays at its end, and the weights of such scores are zero)
                        const float m_new = move ? fmaxf(m_blk, -kFar) : m;
                        const float f = move ? ex2(m - m_new) : 1.f;
                        l *= f;
                        m = m_new;
                        if (j > 0) {
                            wait_product(j - 1);
                            tc_fence_after_sync();
#pragma unroll 1
                            for (int c = 0; c < OWN; c += 32) {
                                uint32_t o[32];
                                tmem_ld_x32(o_col + c, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st_x32(o_col + c, o);
                            }
                        }
                    }
                    // (the buffer that these weights go to is free: the scores of this block were issued, and so have ended, after
                    // the product of two blocks before)
                    // The two tiles take turns on the exponential unit (per scheduler: warps w and w + 4 are on the same one), so
                    // that the loads, maxima and waits of one run beside the exponentials of the other.
                    if (C::TILES == 2 && !SPLIT && (t == 1 || j > 0)) bar_sync(7 + t * 4 + quarter, 64);
                    const float z = m == -INFINITY ? 0.f : m;
                    const float2 c2 = make_float2(scale, scale), z2 = make_float2(-z, -z);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t p[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float2 y = fma2(make_float2(__uint_as_float(x[i][e]), __uint_as_float(x[i][e + 1])), c2, z2);
                            y.x = ex2(y.x);
                            y.y = ex2(y.y);
                            sum[(e / 2) & 1] = add2(sum[(e / 2) & 1], y);
                            p[e / 2] = pack_bf16(y.x, y.y);          // 8 significant bits per weight
                        }
                        tmem_st_x16(s_col + BK + b * (BK / 2) + half * 32 + i * 16, p);
                    }
                    if (C::TILES == 2 && !SPLIT && (t == 0 || j + 1 < mine)) bar_arrive(7 + (t ^ 1) * 4 + quarter, 64);
                    tmem_st_wait();
                    tc_fence_before_sync();
                    if (lane == 0) tell(p_full(t, b));
                    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                }
            };
            if (C::TILES == 2 && split) softmax(std::true_type());
            else softmax(std::false_type());
            // ---- output: with two threads per row each its channels
            if (C::HALVES == 2) l += partner(l);
            wait_product(mine - 1);
            uses[0] += (uint32_t)(mine + 1) / 2;
            uses[1] += (uint32_t)mine / 2;
            tc_fence_after_sync();
            if (split && count > 1) {
                // the second tile's result into the first's (the warps w and w + 4 have the same lanes of tensor memory)
                float2* st = reinterpret_cast<float2*>(stats) + row;
                if (t == 1) {
                    *st = make_float2(m, l);
                    tc_fence_before_sync();
                    bar_sync(1 + quarter, 64);
                    bar_sync(1 + quarter, 64);          // read
                    seq += (long long)count * C::VC;
                    continue;
                }
                bar_sync(1 + quarter, 64);
                tc_fence_after_sync();
                const float2 y = *st;
                const float m_new = fmaxf(m, y.x), z = m_new == -INFINITY ? 0.f : m_new;
                const float f = ex2(m - z), fy = ex2(y.x - z);
                m = m_new;
                l = l * f + y.y * fy;
#pragma unroll 1
                for (int c = 0; c < OWN; c += 32) {
                    uint32_t o[32], v[32];
                    tmem_ld_x32(o_col + c, o);
                    tmem_ld_x32(o_col + D + c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f + __uint_as_float(v[e]) * fy);
                    tmem_st_x32(o_col + c, o);
                }
                tmem_st_wait();
                tc_fence_before_sync();
                bar_sync(1 + quarter, 64);
            }
            // Rows leave in one piece through shared memory (where the queries were: every product with them has ended).
            auto stage = [&](int c, const float (&o)[32], float f) {
#pragma unroll
                for (int e = 0; e < 32; e += 8)
                    sts128(q_place(row, (half * OWN + c + e) / 8),
                           make_uint4(pack_bf16(o[e] * f, o[e + 1] * f), pack_bf16(o[e + 2] * f, o[e + 3] * f),
                                      pack_bf16(o[e + 4] * f, o[e + 5] * f), pack_bf16(o[e + 6] * f, o[e + 7] * f)));
            };
            bool write = true;
            if (it.b0 != 0 || it.b1 != it.blocks) {
                // A part.  Neighbours join in pairs, pairs of pairs and so on, the second to arrive at a pair taking the first
                // one's sum in: log2(parts) steps, each on all SMs that the tile's parts are on, and in an order that does not
                // depend on who arrives when.  [D / 4][ROWS][4 channels], so that the lanes of a warp (rows) lie side by side.
                const Shared sh = shared_by(it, walk.total, workers);
                float* part = a.part_o + (half * OWN * C::ROWS + (part_tile * 128 + row) * 4);
                float2* ml = reinterpret_cast<float2*>(a.part_ml) + part_tile * 128 + row;
                const bool busy = part_tile * 128 + quarter * 32 < live_rows;      // the warp has a row that is one
                int lo = worker - sh.c0;                // this sum: parts lo .. lo + span - 1 (those that there are)
                for (int span = 1; span < sh.parts && write; span *= 2) {
                    const bool right = lo & span;
                    const int other = right ? lo - span : lo + span;
                    if (other >= sh.parts) continue;
                    // (a CTA is the first part of a right side in one tile at most, so its counters name the pair)
                    unsigned* counter = a.counters + 2 * (sh.c0 + (right ? lo : other)) + part_tile;
                    // if the other has arrived, this sum need not be written
                    if (tid == 0) last_flag[t] = others_arrived(counter, 2) ? 1 : 0;
                    bar_sync(5 + t, TILE_THREADS);
                    write = last_flag[t] != 0;
                    if (!write) {
                        const size_t to = (size_t)sh.slot(lo) * C::ROWS;
#pragma unroll 1
                        for (int c = 0; busy && c < OWN; c += 32) {
                            uint32_t o[32];
                            tmem_ld_x32(o_col + c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 32; e += 4)
                                *reinterpret_cast<uint4*>(part + to * D + (c + e) * C::ROWS) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                        }
                        if (half == 0) ml[to] = make_float2(m, l);
                        bar_sync(5 + t, TILE_THREADS);
                        if (tid == 0) last_flag[t] = arrives_last(counter, 2) ? 1 : 0;
                        bar_sync(5 + t, TILE_THREADS);
                        write = last_flag[t] != 0;
                    }
                    if (write) {
                        const size_t from = (size_t)sh.slot(other) * C::ROWS;
                        const float2 y = __ldcg(ml + from);
                        const float m_new = fmaxf(m, y.x), z = m_new == -INFINITY ? 0.f : m_new;
                        const float f = ex2(m - z), fy = ex2(y.x - z);
                        m = m_new;
                        // (no fused multiply: either side may be the one that adds)
                        auto joined = [&](float mine, float theirs) { return __fadd_rn(__fmul_rn(mine, f), __fmul_rn(theirs, fy)); };
                        l = joined(l, y.y);
#pragma unroll 1
                        for (int c = 0; busy && c < OWN; c += 32) {
                            float4 v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = __ldcg(reinterpret_cast<const float4*>(part + from * D + (c + 4 * e) * C::ROWS));
                            uint32_t o[32];
                            tmem_ld_x32(o_col + c, o);
                            tmem_ld_wait();
                            auto add = [&](uint32_t& at, float x) { at = __float_as_uint(joined(__uint_as_float(at), x)); };
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                add(o[4 * e], v[e].x);
                                add(o[4 * e + 1], v[e].y);
                                add(o[4 * e + 2], v[e].z);
                                add(o[4 * e + 3], v[e].w);
                            }
                            tmem_st_x32(o_col + c, o);
                        }
                        tmem_st_wait();
                        bar_sync(5 + t, TILE_THREADS);  // (last_flag is written again)
                    }
                    lo = min(lo, other);
                }
            }
            if (write) {
                l = sum_in_range(m, l, lim);
                const float inv = inverse_sum(l);
#pragma unroll 1
                for (int c = 0; c < OWN; c += 32) {
                    uint32_t o[32];
                    tmem_ld_x32(o_col + c, o);
                    tmem_ld_wait();
                    float f[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(o[e]);
                    stage(c, f, inv);
                }
            }
            if (write) {
                bar_sync(5 + t, TILE_THREADS);
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                    const int at = i * TILE_THREADS + tid, r = at / PIECES, piece = at % PIECES;
                    const int tk = quotient(row0 + r, a.div_g), h = head0 + row0 + r - tk * a.G;
                    if (tk < li.rows_tok)
                        *reinterpret_cast<uint4*>(a.out + ((size_t)(li.q0 + tk) * a.Hq + h) * D + piece * 8) = lds128(q_place(r, piece));
                }
                if (live && half == 0 && a.lse) a.lse[(size_t)(li.q0 + tok) * a.Hq + head0 + row0 + row - tok * a.G] = lse_of(m, l);
            }
            __syncwarp();
            // (the loads above precede this pair's next exchange, and with it the weights that let the next item's
            // product overwrite O)
            tc_fence_before_sync();
            seq += (long long)count * C::VC;
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    if (C::PAIR) cluster_sync();                        // the peer's MMAs and signals reach into this CTA until here
    if (warp == 1) {
        tc_fence_after_sync();
        if (C::PAIR) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && *abort_flag) a.status[0] = (int)EA_ERR_DEVICE_TIMEOUT;
    if (threadIdx.x == 0 && blockIdx.x == 0) *a.operand = 0;
}

template <int D>
ea_status launch(const ea_ctx* ctx, const ea_paged_shape& s, const AttnArgs& args, const void* k_pages, const void* v_pages, cudaStream_t st) {
    using C = Chunk<D>;
    AttnArgs a = args;
    const int sms = ctx->sm_count < kPagedMaxCtas ? ctx->sm_count : kPagedMaxCtas, ctas = C::PAIR ? sms / 2 * 2 : sms;
    a.part_o = static_cast<float*>(ctx->workspace);
    a.part_ml = a.part_o + (size_t)C::PARTS * C::ROWS * D;
    CUtensorMap k_map, v_map;
    const uint32_t kbox = (uint32_t)(s.page_rows < C::KROWS ? s.page_rows : C::KROWS), vbox = (uint32_t)(s.page_rows < C::VKEYS ? s.page_rows : C::VKEYS);
    if (!ea_paged_map(ctx, s, k_pages, kbox, 1, &k_map) || !ea_paged_map(ctx, s, v_pages, vbox, C::VCH / 64, &v_map)) return EA_ERR_CUDA;
    auto kernel = paged_chunk_kernel<D>;
    static std::atomic<uint64_t> done{0};
    ea_status err = ea_allow_smem(kernel, C::SMEM, ctx->device, done);
    if (err != EA_OK) return err;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C::PAIR ? 2 : 1;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    EA_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, k_map, v_map, a));
    ea_count_launches(ctx, 1);
    return EA_CHECK_LAUNCH();
}

}  // namespace

size_t ea_paged_chunk_ws_floats(int d) {
    const int parts = d == 64 ? Chunk<64>::PARTS : d == 128 ? Chunk<128>::PARTS : Chunk<256>::PARTS;
    return (size_t)parts * Chunk<64>::ROWS * (d + 2);
}

ea_status ea_launch_paged_chunk(const ea_ctx* ctx, const ea_paged_shape& s, const AttnArgs& a, const void* k_pages, const void* v_pages,
                                cudaStream_t st) {
    return s.head_dim == 64    ? launch<64>(ctx, s, a, k_pages, v_pages, st)
           : s.head_dim == 128 ? launch<128>(ctx, s, a, k_pages, v_pages, st)
                               : launch<256>(ctx, s, a, k_pages, v_pages, st);
}
