// Attention of new tokens over the paged cache.
//
//   x_{h,i,p} = scale * q_{h,i} . k_{g,p}    for the visible rows p of list g = h / G
//   o_{h,i}   = sum_p e^{x_p - lse} v_{g,p},   lse = log sum_p e^{x_p}
//
// The G query heads that share a list and the new tokens of a sequence are packed into rows, row = token * G + head,
// so that every K/V row is read once for all of them.
#include "paged.h"
#include "paged_attn.cuh"
#include "ptx_sm100.cuh"

using namespace ptx;

namespace {

// ---------------------------------------------------------------------------------------- few rows
// Row tiles of 16: a generation step has G rows per list, and the time is that of reading K and V once.  One CTA per SM
// takes an equal, contiguous share of all key blocks of the call, whatever list they belong to (lengths differ by list);
// a list that several CTAs share is joined by the one of them that ends last.
//
// Inside a CTA one warp keeps TMA boxes of K and V (128-byte swizzle) flowing into a ring, and each of four warps owns 16
// keys of a block: scores (mma.sync m16n8k16, 16 rows are one tile), softmax with its own running maximum, and
// the product with its 16 value rows.  At head_dim <= 128 a second group of four warps takes every other block: a block is a
// chain of some 1300 cycles for a warp, about as long as its bytes take to arrive.  No barrier among the warps until the
// list ends, where they are merged in a fixed order.  At most 16 of the 128 rows of a tcgen05 tile would be in use here,
// and the limit is memory: 32 sequences of up to 16 384 tokens, 28 heads on 4 lists of head_dim 128, 676 MB: 113 us called one
// after the other, 106 in a graph = 6.0 and 6.4 TB/s (0.92 and 0.98 of the measured copy rate); one sequence of 4096 tokens on
// 8 lists, 16.8 MB: 15 and 13 us, most of it the latencies of the share's start, of four blocks per CTA and of the join.
// At head_dim 64 a block takes as long for half the bytes, and the same 676 MB take 140 us = 4.8 TB/s (0.75 of the copy rate).
template <int D> struct Few {
    static constexpr int GROUPS = D == 256 ? 1 : 2;
    static constexpr int NW = 4 * GROUPS;
    static constexpr int BK = 64;                            // keys per block
    static constexpr int CHUNKS = D / 64;
    static constexpr int STAGE = 2 * BK * D * 2;             // K, then V, each box after box: [chunk of 64 channels][row][128 bytes]
    static constexpr int MERGE = NW / 2 * 16 * D * 4;
    // 192 KiB in flight, or nearly; a stage always belongs to the same group, which so waits for each of its uses (a parity
    // tells only neighbouring ones apart)
    static constexpr int NST = (229376 - MERGE) / STAGE / GROUPS * GROUPS;
    static constexpr int THREADS = NW * 32 + 32;
    // behind the ring and the merge buffer: barriers, flags, range, and [NW][16] maxima and sums
    static constexpr int TAIL_ML = 16 * NST + 80;
    static constexpr int TAIL = TAIL_ML + NW * 16 * 8;
    static constexpr int SMEM = 1024 /* alignment */ + NST * STAGE + MERGE + TAIL;
    static_assert(MERGE >= 16 * kPagedMaxCtas * 4, "the weights of the parts fit the merge buffer");
    static_assert(SMEM + 256 <= 232448, "a CTA's shared memory, with room for static arrays");
};

// Joins the parts of a tile of 16 rows, `live` of them in use: THREADS / 16 threads per row turn the parts' maxima and sums into
// weights (in `weight`, [16][parts]), then every thread adds 4 channels of a row over the parts.
template <int D, int THREADS>
__device__ void join_parts(const AttnArgs& a, const Shared& sh, const ListInfo& li, float* weight, int live, int row0, int head0) {
    constexpr int LANES = THREADS / 16, BATCH = D == 256 ? 8 : 16;
    {
        const int row = threadIdx.x / LANES, lane = threadIdx.x % LANES;
        float m = -INFINITY, l = 0.f;
        if (row < live)
            for (int p = lane; p < sh.parts; p += LANES) {
                const float2 v = __ldcg(reinterpret_cast<const float2*>(a.part_ml) + (size_t)sh.slot(p) * 16 + row);
                const float top = fmaxf(m, v.x), z = top == -INFINITY ? 0.f : top;
                l = l * ex2(m - z) + v.y * ex2(v.x - z);
                m = top;
                weight[row * kPagedMaxCtas + p] = v.x;
            }
        float top = m;
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float z = top == -INFINITY ? 0.f : top;
        l *= ex2(m - z);
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        if (row < live) {
            const int tok = quotient(row0 + row, a.div_g);
            l = sum_in_range(top, l, limit_of(li, a, tok));
            const float inv = inverse_sum(l);
            for (int p = lane; p < sh.parts; p += LANES) weight[row * kPagedMaxCtas + p] = ex2(weight[row * kPagedMaxCtas + p] - z) * inv;
            if (lane == 0 && a.lse) a.lse[(size_t)(li.q0 + tok) * a.Hq + head0 + row0 + row - tok * a.G] = lse_of(top, l);
        }
    }
    bar_sync(1, THREADS);
    const int bits = live > 8 ? 4 : live > 4 ? 3 : live > 2 ? 2 : live - 1;
    for (int i = threadIdx.x; i < (D / 4) << bits; i += THREADS) {
        const int row = i & ((1 << bits) - 1), col = (i >> bits) * 4;
        if (row >= live) continue;
        const float* src = a.part_o + (col * 16) + row * 4;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int b = 0; b < sh.parts; b += BATCH) {      // so many loads on their way at a time
            float4 v[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (b + k < sh.parts) v[k] = __ldcg(reinterpret_cast<const float4*>(src + (size_t)sh.slot(b + k) * 16 * D));
            }
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float w = b + k < sh.parts ? weight[row * kPagedMaxCtas + b + k] : 0.f;
                o.x += v[k].x * w;
                o.y += v[k].y * w;
                o.z += v[k].z * w;
                o.w += v[k].w * w;
            }
        }
        const int tok = quotient(row0 + row, a.div_g);
        const size_t at = (size_t)(li.q0 + tok) * a.Hq + head0 + row0 + row - tok * a.G;
        *reinterpret_cast<uint2*>(a.out + at * D + col) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
    }
}

template <int D>
__global__ void __launch_bounds__(Few<D>::THREADS, 1)
paged_few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const AttnArgs a) {
    using C = Few<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
    float* merge = reinterpret_cast<float*>(gen + C::NST * C::STAGE);
    uint8_t* tail = gen + C::NST * C::STAGE + C::MERGE;
    const uint32_t bars = base + C::NST * C::STAGE + C::MERGE;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (C::NST + s); };
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 16 * C::NST);
    Walk* start = reinterpret_cast<Walk*>(tail + 16 * C::NST + 16);
    float* ml = reinterpret_cast<float*>(tail + C::TAIL_ML);                             // [NW][16][2]
    static_assert(16 + sizeof(Walk) <= 80, "flags and range fit before the maxima");
    volatile int* last_flag = abort_flag + 1;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::NST; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 4);
        }
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&k_map);
        prefetch_tensormap(&v_map);
    }
    find_range<C::THREADS>(a, C::BK, 16, blockIdx.x, gridDim.x, start);
    __syncthreads();
    Walk walk = *start;
    Item it;
    long long block_no = 0;
    bool ok = true;

    if (warp == C::NW) {
        // ------------------------------------------------------------------------------ producer
        const int box_shift = a.shift < 6 ? a.shift : 6;                 // rows per box: a page, at most 64
        const int box_rows = 1 << box_shift;
        const int subs = C::BK >> box_shift;
        const uint32_t leader = elect_one();
        const uint64_t policy = evict_first_policy();                    // every row is read once (676 MB behind a write of all of L2: 142 -> 127 us)
        while (next_item(a, walk, 16, C::BK, it)) {
            const ListInfo& li = it.li;
            const int r = it.list, b0 = it.b0;
            const int entries = (int)(((unsigned)li.n + (1u << a.shift) - 1u) >> a.shift);
            const int32_t* tab = a.table + (size_t)r * a.max_pages;
            // table entries ride in registers, 32 ahead of the 32 in use
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
            int win = ((b0 * C::BK) >> a.shift) & ~31;
            int cur = entry(win + lane), next = entry(win + 32 + lane);
            for (int b = b0; b < it.b1; ++b, ++block_no) {
                const int s = (int)(block_no % C::NST);
                const uint32_t use = (uint32_t)(block_no / C::NST);
                const int e0 = (b * C::BK) >> a.shift;
                if (e0 >= win + 32) {
                    win += 32;
                    cur = next;
                    next = entry(win + 32 + lane);
                }
                if (ok) ok = mbar_wait(empty(s), (use & 1) ^ 1, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) continue;
                const int rest = li.n - b * C::BK;
                int act = rest <= 0 ? 0 : (rest + box_rows - 1) >> box_shift;
                if (act > subs) act = subs;
                if (leader) mbar_arrive_expect_tx(full(s), (uint32_t)(act * C::CHUNKS * 2 * box_rows * 128));
                __syncwarp();
                const uint32_t to = base + (uint32_t)(s * C::STAGE);
                int y[4];                                       // first row of each box in the pool
#pragma unroll
                for (int sub = 0; sub < 4; ++sub) {
                    const int key = b * C::BK + (sub << box_shift);
                    const int page = __shfl_sync(0xffffffffu, cur, ((key >> a.shift) - win) & 31);
                    y[sub] = (page << a.shift) + (key & ((1 << a.shift) - 1));
                }
#pragma unroll
                for (int sub = 0; sub < 4; ++sub)
                    if (sub < act) {
                        const uint32_t at = to + (uint32_t)(sub * D * 2) * (uint32_t)box_rows;
                        tma_load_3d_warp(leader, at, &k_map, full(s), 0, y[sub], 0, policy);
                        tma_load_3d_warp(leader, at + C::STAGE / 2, &v_map, full(s), 0, y[sub], 0, policy);
                    }
            }
        }
        if (!ok && lane == 0) {
            // copies in flight land before the shared memory goes away
            for (int s = 0; s < C::NST; ++s) {
                mbar_drain(full(s), 0);
                mbar_drain(full(s), 1);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------------------ consumers
        const int g8 = lane >> 2, t4 = lane & 3;
        // ldmatrix row addresses inside a stage (K: keys by channels; V: transposed on the way)
        const int lm = lane >> 3, lr = lane & 7;
        const int group = warp / 4, slice = warp % 4 * 16;
        const int box_shift = a.shift < 6 ? a.shift : 6;
        const uint32_t chunk_bytes = 128u << box_shift;         // 64 channels of a box
        const uint32_t box_off = (uint32_t)(slice >> box_shift) * C::CHUNKS * chunk_bytes + (uint32_t)(slice & ((1 << box_shift) - 1)) * 128u;
        const uint32_t k_row = box_off + (uint32_t)((lm >> 1) * 8 + lr) * 128u;
        const uint32_t v_row = box_off + (uint32_t)((lm & 1) * 8 + lr) * 128u;
        const uint32_t sw = (uint32_t)lr << 4;
        while (next_item(a, walk, 16, C::BK, it)) {
            const ListInfo& li = it.li;
            const int tile = it.tile, b0 = it.b0;
            const int head0 = (it.list - quotient(it.list, a.div_hkv) * a.Hkv) * a.G;
            // rows g8 and g8 + 8 of the tile
            int tok[2], hd[2], lim[2];
            bool live[2];
            uint32_t qf[D / 16][4];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int pr = tile * 16 + g8 + 8 * x;
                tok[x] = quotient(pr, a.div_g);
                hd[x] = head0 + pr - tok[x] * a.G;
                live[x] = tok[x] < li.rows_tok;
                lim[x] = live[x] ? limit_of(li, a, tok[x]) : 0;
                const __nv_bfloat16* src = a.q + (long long)(li.q0 + (live[x] ? tok[x] : 0)) * a.q_stride + (long long)hd[x] * D;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    qf[ks][x] = live[x] ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + t4 * 2) : 0u;
                    qf[ks][x + 2] = live[x] ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + 8 + t4 * 2) : 0u;
                }
            }
            float o[D / 8][4];
#pragma unroll
            for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
            float mx[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};

            for (int b = b0; b < it.b1; ++b, ++block_no) {
                const int s = (int)(block_no % C::NST);
                const uint32_t use = (uint32_t)(block_no / C::NST);
                if (C::GROUPS == 2 && (block_no & 1) != group) continue;
                if (ok) ok = mbar_wait(full(s), use & 1, abort_flag);
                const int key0 = b * C::BK + slice;
                if (key0 < li.n) {
                    const uint32_t ks_base = base + (uint32_t)(s * C::STAGE);
                    float x0[4] = {0.f, 0.f, 0.f, 0.f}, x1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        uint32_t kf[4];
                        const uint32_t col = (uint32_t)((ks % 4) * 32 + (lm & 1) * 16);
                        ldmatrix_x4(ks_base + (ks / 4) * chunk_bytes + k_row + (col ^ sw), kf);
                        mma_bf16(x0, qf[ks], kf[0], kf[1]);
                        mma_bf16(x1, qf[ks], kf[2], kf[3]);
                    }
                    const int ka = key0 + t4 * 2;
                    float y[2][4];
                    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        y[x][0] = ka < lim[x] ? x0[2 * x] * a.scale_log2 : -INFINITY;
                        y[x][1] = ka + 1 < lim[x] ? x0[2 * x + 1] * a.scale_log2 : -INFINITY;
                        y[x][2] = ka + 8 < lim[x] ? x1[2 * x] * a.scale_log2 : -INFINITY;
                        y[x][3] = ka + 9 < lim[x] ? x1[2 * x + 1] * a.scale_log2 : -INFINITY;
                        top[x] = fmaxf(fmaxf(y[x][0], y[x][1]), fmaxf(y[x][2], y[x][3]));
                        top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 1));
                        top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 2));
                    }
                    if (__any_sync(0xffffffffu, top[0] > mx[0] || top[1] > mx[1])) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float m_new = fmaxf(mx[x], top[x]);
                            const float f = m_new == -INFINITY ? 1.f : ex2(mx[x] - m_new);
                            mx[x] = m_new;
                            sum[x] *= f;
#pragma unroll
                            for (int i = 0; i < D / 8; ++i) {
                                o[i][2 * x] *= f;
                                o[i][2 * x + 1] *= f;
                            }
                        }
                    }
                    uint32_t pf[4];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float z = mx[x] == -INFINITY ? 0.f : mx[x];          // a row that has seen no key yet
                        // (of the rounded products, all four alike, and not fused with them)
                        const float p0 = ex2(__fsub_rn(y[x][0], z)), p1 = ex2(__fsub_rn(y[x][1], z));
                        const float p2 = ex2(__fsub_rn(y[x][2], z)), p3 = ex2(__fsub_rn(y[x][3], z));
                        sum[x] += (p0 + p1) + (p2 + p3);
                        pf[x] = pack_bf16(p0, p1);           // the weights enter the product with 8 significant bits
                        pf[x + 2] = pack_bf16(p2, p3);
                    }
                    const uint32_t vs_base = ks_base + C::STAGE / 2;
                    // rows behind the list's end hold anything: a weight of zero does not silence a NaN
                    uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
                    if (key0 + 16 > li.n) {
                        keep0 = (ka < li.n ? 0xffffu : 0u) | (ka + 1 < li.n ? 0xffff0000u : 0u);
                        keep1 = (ka + 8 < li.n ? 0xffffu : 0u) | (ka + 9 < li.n ? 0xffff0000u : 0u);
                    }
#pragma unroll
                    for (int nt = 0; nt < D / 16; ++nt) {
                        uint32_t vf[4];
                        const uint32_t col = (uint32_t)((nt % 4) * 32 + (lm >> 1) * 16);
                        ldmatrix_x4_trans(vs_base + (nt / 4) * chunk_bytes + v_row + (col ^ sw), vf);
                        mma_bf16(o[2 * nt], pf, vf[0] & keep0, vf[1] & keep1);
                        mma_bf16(o[2 * nt + 1], pf, vf[2] & keep0, vf[3] & keep1);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(s));
            }

            // the warps' shares of the list: one maximum, then a tree of additions in a fixed order
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                sum[x] += __shfl_xor_sync(0xffffffffu, sum[x], 1);
                sum[x] += __shfl_xor_sync(0xffffffffu, sum[x], 2);
                if (t4 == 0) {
                    ml[(warp * 16 + g8 + 8 * x) * 2] = mx[x];
                    ml[(warp * 16 + g8 + 8 * x) * 2 + 1] = sum[x];
                }
            }
            bar_sync(1, C::NW * 32);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float m_all = -INFINITY, l_all = 0.f;
#pragma unroll
                for (int w = 0; w < C::NW; ++w) m_all = fmaxf(m_all, ml[(w * 16 + g8 + 8 * x) * 2]);
                const float z = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
                for (int w = 0; w < C::NW; ++w) l_all += ml[(w * 16 + g8 + 8 * x) * 2 + 1] * ex2(ml[(w * 16 + g8 + 8 * x) * 2] - z);
                const float f = ex2(mx[x] - z);
                mx[x] = m_all;
                sum[x] = l_all;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    o[i][2 * x] *= f;
                    o[i][2 * x + 1] *= f;
                }
            }
            const bool upper = li.rows_tok * a.G - tile * 16 > 8;       // rows 8-15 of the tile are in use
#pragma unroll
            for (int h = C::NW / 2; h >= 1; h /= 2) {
                if (warp >= h && warp < 2 * h) {
                    float2* dst = reinterpret_cast<float2*>(merge) + (size_t)(h == C::NW / 2 ? warp - h : warp) * (D / 8) * 64 + lane;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) dst[i * 64] = make_float2(o[i][0], o[i][1]);
                    if (upper)
#pragma unroll
                        for (int i = 0; i < D / 8; ++i) dst[i * 64 + 32] = make_float2(o[i][2], o[i][3]);
                }
                bar_sync(1, C::NW * 32);
                if (warp < h) {
                    const float2* src = reinterpret_cast<const float2*>(merge) + (size_t)(h == C::NW / 2 ? warp : warp + h) * (D / 8) * 64 + lane;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        const float2 v = src[i * 64];
                        o[i][0] += v.x;
                        o[i][1] += v.y;
                    }
                    if (upper)
#pragma unroll
                        for (int i = 0; i < D / 8; ++i) {
                            const float2 v = src[i * 64 + 32];
                            o[i][2] += v.x;
                            o[i][3] += v.y;
                        }
                }
            }
            const bool whole = b0 == 0 && it.b1 == it.blocks;
            if (whole) {
                if (warp != 0) continue;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!live[x]) continue;
                    sum[x] = sum_in_range(mx[x], sum[x], lim[x]);
                    const float inv = inverse_sum(sum[x]);
                    const size_t row = (size_t)(li.q0 + tok[x]) * a.Hq + hd[x];
                    uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * D) + t4;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) dst[i * 4] = pack_bf16(o[i][2 * x] * inv, o[i][2 * x + 1] * inv);
                    if (a.lse && t4 == 0) a.lse[row] = lse_of(mx[x], sum[x]);
                }
                continue;
            }
            const Shared sh = shared_by(it, walk.total, gridDim.x);
            if (warp == 0) {
                const size_t slot = (size_t)2 * blockIdx.x + (it.first ? 0 : 1);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!live[x]) continue;
                    // (a part: [D / 4][16 rows][4 channels])
                    float2* dst = reinterpret_cast<float2*>(a.part_o + slot * 16 * D + ((t4 / 2) * 16 + g8 + 8 * x) * 4 + (t4 & 1) * 2);
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) dst[i * 64] = make_float2(o[i][2 * x], o[i][2 * x + 1]);
                    if (t4 == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * 16 + g8 + 8 * x) * 2) = make_float2(mx[x], sum[x]);
                }
                __syncwarp();
                if (lane == 0) *last_flag = arrives_last(a.counters + sh.c0, sh.parts) ? 1 : 0;
            }
            bar_sync(1, C::NW * 32);
            if (*last_flag)
                join_parts<D, C::NW * 32>(a, sh, li, merge, min(16, li.rows_tok * a.G - tile * 16), tile * 16, head0);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) a.status[0] = (int)EA_ERR_DEVICE_TIMEOUT;
    if (threadIdx.x == 0 && blockIdx.x == 0) *a.operand = 0;
}

size_t few_part_floats(int d) { return (size_t)2 * kPagedMaxCtas * 16 * (d + 2); }

template <int D>
ea_status launch_few(const ea_ctx* ctx, const ea_paged_shape& s, const AttnArgs& args, const void* k_pages, const void* v_pages,
                     cudaStream_t st) {
    using C = Few<D>;
    AttnArgs a = args;
    const int ctas = ctx->sm_count < kPagedMaxCtas ? ctx->sm_count : kPagedMaxCtas;
    a.part_o = static_cast<float*>(ctx->workspace);
    a.part_ml = a.part_o + (size_t)2 * kPagedMaxCtas * 16 * D;
    CUtensorMap k_map, v_map;
    const uint32_t box = s.page_rows < 64 ? (uint32_t)s.page_rows : 64u;
    if (!ea_paged_map(ctx, s, k_pages, box, D / 64, &k_map) || !ea_paged_map(ctx, s, v_pages, box, D / 64, &v_map)) return EA_ERR_CUDA;
    auto kernel = paged_few_kernel<D>;
    static std::atomic<uint64_t> done{0};
    ea_status err = ea_allow_smem(kernel, C::SMEM, ctx->device, done);
    if (err != EA_OK) return err;
    kernel<<<ctas, C::THREADS, C::SMEM, st>>>(k_map, v_map, a);
    ea_count_launches(ctx, 1);
    return EA_CHECK_LAUNCH();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

bool ea_paged_map(const ea_ctx* ctx, const ea_paged_shape& s, const void* pages, uint32_t rows, uint32_t chunks, CUtensorMap* map) {
    // an empty pool is never read (list_info refuses every row of it), but a map needs an address and a size
    const uint64_t n = (uint64_t)(s.n_pages > 0 ? s.n_pages : 1) * (uint64_t)s.page_rows;
    return ea_tensor_map_bf16_3d(map, s.n_pages > 0 ? pages : ctx->workspace, 64, n, (uint64_t)s.head_dim / 64, (uint64_t)s.head_dim * 2,
                                 128, 64, rows, false, chunks);
}

// Up to 16 rows per list fit one tile of the kernel for few rows; more go to the tensor-core tiles of 128.  Both at 16 rows
// of 128 lists of 8192 keys: head_dim 64 60 against 75 us, 128 101 against 115, 256 184 against 201; of 8 lists: 128 27 against
// 42.  At 20 rows, where this kernel reads everything twice, 128 lists: 184 against 115 at head_dim 128, 348 against 201 at 256.
static bool few_rows(int max_q, int G) { return (long long)max_q * G <= 16; }

size_t ea_paged_attn_ws_bytes(const ea_paged_shape& s, int max_q) {
    const size_t few = few_part_floats(s.head_dim);
    return (few_rows(max_q, s.n_q_heads / s.n_kv_heads) ? few : ea_paged_chunk_ws_floats(s.head_dim)) * sizeof(float);
}

extern "C" ea_status ea_paged_attention(ea_ctx* ctx, const ea_paged_shape* shape, const void* q, int64_t q_stride, int32_t n_tokens,
                                        const int32_t* q_offsets, int32_t max_q, const int32_t* kv_lens, const int32_t* block_table,
                                        const void* k_pages, const void* v_pages, float scale, int32_t causal, void* out,
                                        float* lse_opt, void* cuda_stream) {
    if (!ctx) return EA_ERR_INVALID_ARG;
    ea_status st = ea_check_paged_shape(shape);
    if (st != EA_OK) return st;
    if (n_tokens < 0 || max_q < 0 || max_q > n_tokens || !(fabsf(scale) <= 2.0e38f)) return EA_ERR_INVALID_ARG;
    const int64_t dense = (int64_t)shape->n_q_heads * shape->head_dim;
    if (q_stride == 0) q_stride = dense;
    if (q_stride < dense || q_stride % 8 != 0) return EA_ERR_INVALID_ARG;
    if ((int64_t)n_tokens * shape->n_q_heads > 0x7fffffffLL) return EA_ERR_UNSUPPORTED;
    if (shape->n_seqs == 0 || n_tokens == 0 || max_q == 0) return EA_OK;
    if (!q || !q_offsets || !kv_lens || !out || (shape->max_pages > 0 && !block_table)) return EA_ERR_INVALID_ARG;
    if (shape->n_pages > 0 && (!k_pages || !v_pages)) return EA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned4(q_offsets) || !aligned4(kv_lens) ||
        !aligned4(block_table) || !aligned4(lse_opt))
        return EA_ERR_INVALID_ARG;
    if (ctx->workspace_bytes < ea_paged_attn_ws_bytes(*shape, max_q)) return EA_ERR_WORKSPACE;
    const long long lists = (long long)shape->n_seqs * shape->n_kv_heads;
    const long long pool = (long long)shape->n_pages * shape->page_rows * shape->head_dim * 2;
    const Span spans[] = {{q, 2 * ((n_tokens - 1) * q_stride + dense), false}, {q_offsets, (shape->n_seqs + 1LL) * 4, false},
                          {kv_lens, lists * 4, false}, {block_table, lists * shape->max_pages * 4, false}, {k_pages, pool, false},
                          {v_pages, pool, false}, {out, 2 * n_tokens * dense, true},
                          {lse_opt, 4LL * n_tokens * shape->n_q_heads, true}};
    if (outputs_overlap(spans)) return EA_ERR_INVALID_ARG;
    AttnArgs a = {};
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.q_stride = q_stride;
    a.q_off = q_offsets;
    a.kv_len = kv_lens;
    a.table = block_table;
    a.out = static_cast<__nv_bfloat16*>(out);
    a.lse = lse_opt;
    a.status = ctx->status_dev;
    a.counters = ctx->counters;
    a.operand = ea_operand_word(ctx);
    a.lists = shape->n_seqs * shape->n_kv_heads;
    a.Hq = shape->n_q_heads;
    a.Hkv = shape->n_kv_heads;
    a.G = shape->n_q_heads / shape->n_kv_heads;
    a.shift = __builtin_ctz((unsigned)shape->page_rows);
    a.n_pages = shape->n_pages;
    a.max_pages = shape->max_pages;
    a.n_tokens = n_tokens;
    a.max_q = max_q;
    a.causal = causal != 0;
    a.div_g = fast_div(a.G);
    a.div_hkv = fast_div(a.Hkv);
    a.scale_log2 = scale * 1.4426950408889634f;
    int prev = 0;
    EA_CUDA_TRY(cudaGetDevice(&prev));
    if (prev != ctx->device) EA_CUDA_TRY(cudaSetDevice(ctx->device));
    ctx->image_ready = false;                       // the partial results lie where fused statistics keep their images
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!few_rows(max_q, a.G))
        st = ea_launch_paged_chunk(ctx, *shape, a, k_pages, v_pages, stream);
    else
        st = shape->head_dim == 64    ? launch_few<64>(ctx, *shape, a, k_pages, v_pages, stream)
             : shape->head_dim == 128 ? launch_few<128>(ctx, *shape, a, k_pages, v_pages, stream)
                                      : launch_few<256>(ctx, *shape, a, k_pages, v_pages, stream);
    if (prev != ctx->device) cudaSetDevice(prev);
    return st;
}
