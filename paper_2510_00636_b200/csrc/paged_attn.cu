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
// a list that several CTAs share leaves partial results (maximum, sum, unnormalised output) for paged_combine_kernel.
//
// Inside a CTA one warp keeps TMA boxes of K and V (128-byte swizzle) flowing into a ring, and each of four warps owns 16
// keys of a block: scores (mma.sync m16n8k16, 16 rows are one tile), softmax with its own running maximum, and
// the product with its 16 value rows.  At head_dim <= 128 a second group of four warps takes every other block: a block is a
// chain of some 1300 cycles for a warp, about as long as its bytes take to arrive.  No barrier among the warps until the
// list ends, where they are merged in a fixed order.  At most 16 of the 128 rows of a tcgen05 tile would be in use here,
// and the limit is memory.
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
    // behind the ring and the merge buffer: barriers, abort flag, range, and [NW][16] maxima and sums
    static constexpr int TAIL_ML = 16 * NST + 64;
    static constexpr int TAIL = TAIL_ML + NW * 16 * 8;
    static constexpr int SMEM = 1024 /* alignment */ + NST * STAGE + MERGE + TAIL;
    static_assert(SMEM + 256 <= 232448, "a CTA's shared memory, with room for static arrays");
};

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
    static_assert(16 + sizeof(Walk) <= 64, "flag and range fit before the maxima");

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
        const uint64_t policy = evict_first_policy();                    // every row is read once: 142 -> 127 us for 676 MB
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
                        const float p0 = ex2(y[x][0] - z), p1 = ex2(y[x][1] - z), p2 = ex2(y[x][2] - z), p3 = ex2(y[x][3] - z);
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
#pragma unroll
            for (int h = C::NW / 2; h >= 1; h /= 2) {
                if (warp >= h && warp < 2 * h) {
                    float4* dst = reinterpret_cast<float4*>(merge) + (size_t)(h == C::NW / 2 ? warp - h : warp) * (D / 8) * 32 + lane;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) dst[i * 32] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
                }
                bar_sync(1, C::NW * 32);
                if (warp < h) {
                    const float4* src = reinterpret_cast<const float4*>(merge) + (size_t)(h == C::NW / 2 ? warp : warp + h) * (D / 8) * 32 + lane;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        const float4 v = src[i * 32];
                        o[i][0] += v.x;
                        o[i][1] += v.y;
                        o[i][2] += v.z;
                        o[i][3] += v.w;
                    }
                }
            }
            if (warp == 0) {
                const bool whole = b0 == 0 && it.b1 == it.blocks;
                const size_t slot = 2 * (size_t)blockIdx.x + (it.first ? 0 : 1);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!live[x]) continue;
                    if (whole) {
                        const float inv = sum[x] > 0.f ? 1.f / sum[x] : (sum[x] == 0.f ? 0.f : sum[x]);
                        const size_t row = (size_t)(li.q0 + tok[x]) * a.Hq + hd[x];
                        uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * D) + t4;
#pragma unroll
                        for (int i = 0; i < D / 8; ++i) dst[i * 4] = pack_bf16(o[i][2 * x] * inv, o[i][2 * x + 1] * inv);
                        if (a.lse && t4 == 0) a.lse[row] = lse_of(mx[x], sum[x]);
                    } else {
                        // (parts: [D / 4][16 rows][4 channels])
                        float2* dst = reinterpret_cast<float2*>(a.part_o + slot * 16 * D + ((t4 / 2) * 16 + g8 + 8 * x) * 4 + (t4 & 1) * 2);
#pragma unroll
                        for (int i = 0; i < D / 8; ++i) dst[i * 64] = make_float2(o[i][2 * x], o[i][2 * x + 1]);
                        if (t4 == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * 16 + g8 + 8 * x) * 2) = make_float2(mx[x], sum[x]);
                    }
                }
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) a.status[0] = (int)EA_ERR_DEVICE_TIMEOUT;
}

// Joins the partial results of row tiles (ROWS rows) that several CTAs shared: one CTA per (tile, 16 of its rows, list).
// First a warp per row turns the parts' maxima and sums into weights, then every thread adds 4 channels of a row over
// the parts, in the order of the keys.
template <int D, int ROWS>
__global__ void __launch_bounds__(128) paged_combine_kernel(const AttnArgs a, int BK, int ctas) {
    __shared__ float weight[16][kPagedMaxCtas];
    constexpr int GROUPS = ROWS / 16;
    const int r = blockIdx.y, tile = blockIdx.x / GROUPS, row0 = blockIdx.x % GROUPS * 16;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const ListInfo li = list_info(a, r, false);
    const int head0 = (r - quotient(r, a.div_hkv) * a.Hkv) * a.G;
    const int rows_left = li.rows_tok * a.G - (tile * ROWS + row0);
    if (rows_left <= 0) return;
    const int live = min(rows_left, 16);
    long long before, total;
    count_units<128>(a, BK, ROWS, r, &before, &total);
    long long u0 = before;
    for (int t = 0; t < tile; ++t) u0 += tile_blocks(li, a, t, ROWS, BK);
    const long long u1 = u0 + tile_blocks(li, a, tile, ROWS, BK);
    const Division division(total, ctas);
    const int c0 = division.owner(u0), c1 = division.owner(u1 - 1), parts = c1 - c0 + 1;
    if (parts == 1) return;
    // a CTA's first item is its part 0, its last part 1: only the tile's first CTA may have begun before it
    const size_t p0 = ((size_t)2 * c0 + (u0 > division.begin(c0) ? 1 : 0)) * ROWS + row0;
    const size_t p1 = (size_t)2 * (c0 + 1) * ROWS + row0;                   // part 1 of the tile; the next ones 2 ROWS on
    for (int row = warp; row < live; row += 4) {
        float m = -INFINITY, l = 0.f;
        for (int p = lane; p < parts; p += 32) {
            const float2 v = *reinterpret_cast<const float2*>(a.part_ml + ((p == 0 ? p0 : p1 + (size_t)(p - 1) * 2 * ROWS) + row) * 2);
            weight[row][p] = v.x;
            m = fmaxf(m, v.x);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        const float z = m == -INFINITY ? 0.f : m;
        for (int p = lane; p < parts; p += 32) {
            const float f = ex2(weight[row][p] - z);
            l += f * a.part_ml[((p == 0 ? p0 : p1 + (size_t)(p - 1) * 2 * ROWS) + row) * 2 + 1];
            weight[row][p] = f;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
        for (int p = lane; p < parts; p += 32) weight[row][p] *= inv;
        if (lane == 0 && a.lse) {
            const int pr = tile * ROWS + row0 + row, tok = quotient(pr, a.div_g);
            a.lse[(size_t)(li.q0 + tok) * a.Hq + head0 + pr - tok * a.G] = lse_of(m, l);
        }
    }
    __syncthreads();
    // (a part's rows lie side by side in pieces of 4 channels: [D / 4][ROWS][4])
    const int bits = live > 8 ? 4 : live > 4 ? 3 : live > 2 ? 2 : live - 1;
    for (int i = threadIdx.x; i < (D / 4) << bits; i += 128) {
        const int row = i & ((1 << bits) - 1), col = (i >> bits) * 4;
        if (row >= live) continue;
        const float* src = a.part_o + (p0 - row0) * D + (size_t)(col * ROWS) + (row0 + row) * 4;
        const float* next = a.part_o + (p1 - row0) * D + (size_t)(col * ROWS) + (row0 + row) * 4;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int b = 0; b < parts; b += 8) {             // eight loads on their way at a time
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (b + k < parts) v[k] = __ldcg(reinterpret_cast<const float4*>(b + k == 0 ? src : next + (size_t)(b + k - 1) * 2 * ROWS * D));
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float w = b + k < parts ? weight[row][b + k] : 0.f;
                o.x += v[k].x * w;
                o.y += v[k].y * w;
                o.z += v[k].z * w;
                o.w += v[k].w * w;
            }
        }
        const int pr = tile * ROWS + row0 + row, tok = quotient(pr, a.div_g);
        const size_t at = (size_t)(li.q0 + tok) * a.Hq + head0 + pr - tok * a.G;
        *reinterpret_cast<uint2*>(a.out + at * D + col) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
    }
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
    err = EA_CHECK_LAUNCH();
    if (err != EA_OK) return err;
    return ea_launch_paged_combine(ctx, s, a, 16, C::BK, ctas, st);
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

ea_status ea_launch_paged_combine(const ea_ctx* ctx, const ea_paged_shape& s, const AttnArgs& a, int rows, int BK, int ctas, cudaStream_t st) {
    const dim3 grid((unsigned)(((long long)a.max_q * a.G + rows - 1) / rows * (rows / 16)), (unsigned)(s.n_seqs * s.n_kv_heads));
    const int d = s.head_dim;
    auto kernel = rows == 16    ? (d == 64 ? paged_combine_kernel<64, 16> : d == 128 ? paged_combine_kernel<128, 16> : paged_combine_kernel<256, 16>)
                  : rows == 128 ? paged_combine_kernel<256, 128>
                                : (d == 64 ? paged_combine_kernel<64, 256> : paged_combine_kernel<128, 256>);
    kernel<<<grid, 128, 0, st>>>(a, BK, ctas);
    ea_count_launches(ctx, 1);
    return EA_CHECK_LAUNCH();
}

// Up to 16 rows per list fit one tile of the kernel for few rows; more go to the tensor-core tiles of 128.
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
    if (n_tokens < 0 || max_q < 0 || max_q > n_tokens || !(fabsf(scale) <= 3.0e38f)) return EA_ERR_INVALID_ARG;
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
    AttnArgs a = {};
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.q_stride = q_stride;
    a.q_off = q_offsets;
    a.kv_len = kv_lens;
    a.table = block_table;
    a.out = static_cast<__nv_bfloat16*>(out);
    a.lse = lse_opt;
    a.status = ctx->status_dev;
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
