// What the attention kernels over the paged cache share: the description of a list, the division of the call's key
// blocks among the CTAs, and small wrappers.
#pragma once

#include <cuda_bf16.h>

#include "ea_internal.h"
#include "fast_div.cuh"
#include "paged.h"

struct AttnArgs {
    const __nv_bfloat16* q;
    long long q_stride;          // elements between tokens
    const int32_t* q_off;        // [n_seqs + 1]
    const int32_t* kv_len;       // [lists]
    const int32_t* table;        // [lists][max_pages]
    __nv_bfloat16* out;          // [n_tokens, Hq, d]
    float* lse;                  // [n_tokens, Hq] or nullptr
    float* part_o;               // unnormalised partial outputs, two row tiles per CTA
    float* part_ml;              // their maxima (of scores in units of log 2) and sums
    unsigned* counters;          // arrivals at the row tiles that several CTAs share
    unsigned* operand;           // the parts lie where a fused statistics operand would
    int* status;
    int lists, Hq, Hkv, G, shift, n_pages, max_pages, n_tokens, max_q, causal;
    FastDiv div_g, div_hkv;      // by G and by Hkv
    float scale_log2;
};

struct ListInfo {
    int m;                       // new tokens of the sequence
    int rows_tok;                // of them, those that the call serves (max_q at most)
    int q0;                      // the first one's row in q
    int n;                       // rows of the list
};

// Lengths and offsets live on the device, so they are checked here: what does not fit is reported and left out.
__device__ __forceinline__ ListInfo list_info(const AttnArgs& a, int r, bool report) {
    const int s = quotient(r, a.div_hkv);
    const int q0 = a.q_off[s], q1 = a.q_off[s + 1];
    ListInfo li = {0, 0, 0, 0};
    bool bad = q0 < 0 || q1 < q0 || q1 > a.n_tokens;
    if (!bad) {
        li.m = q1 - q0;
        li.q0 = q0;
        li.rows_tok = li.m < a.max_q ? li.m : a.max_q;
        bad = li.m > a.max_q;
    }
    const long long cap = a.n_pages > 0 ? (long long)a.max_pages << a.shift : 0;
    int n = a.kv_len[r];
    if (n < 0 || n > cap) {
        bad = true;
        n = n < 0 ? 0 : (int)cap;
    }
    li.n = n;
    if (bad && report) a.status[1] = (int)EA_ERR_PAGES;
    return li;
}
// (packed rows of a call are below 2^31: n_tokens * Hq is)
__device__ __forceinline__ int tiles_of(const ListInfo& li, const AttnArgs& a, int rows) { return (int)(((unsigned)(li.rows_tok * a.G) + rows - 1u) / (unsigned)rows); }
// First row of a list that token `tok` does not see.
__device__ __forceinline__ int limit_of(const ListInfo& li, const AttnArgs& a, int tok) {
    if (!a.causal) return li.n;
    const int v = li.n - li.m + tok + 1;                 // tok < m: between -2^31 and n
    return v < 0 ? 0 : v;
}
// Key blocks that a row tile looks at: one at least, so that rows which see nothing still have their outputs written.
__device__ __forceinline__ int tile_blocks(const ListInfo& li, const AttnArgs& a, int tile, int rows, int BK) {
    const int end = min((tile + 1) * rows, li.rows_tok * a.G);
    const int lim = limit_of(li, a, quotient(end - 1, a.div_g));
    return lim > BK ? (int)(((unsigned)lim + BK - 1u) / BK) : 1;
}
__device__ __forceinline__ long long list_units(const ListInfo& li, const AttnArgs& a, int rows, int BK) {
    const int tiles = tiles_of(li, a, rows);
    long long u = 0;
    for (int t = 0; t < tiles; ++t) u += tile_blocks(li, a, t, rows, BK);
    return u;
}

// The call's W units (unit: one key block of one row tile) in their order, divided among n CTAs: W / n each and one more
// for the first W mod n, so that the owners of consecutive units are consecutive CTAs, none of them idle.
struct Division {
    long long each;
    int extra;
    __device__ __forceinline__ Division(long long total, int ctas) : each(total / ctas), extra((int)(total % ctas)) {}
    __device__ __forceinline__ long long begin(int c) const { return c * each + (c < extra ? c : extra); }
    __device__ __forceinline__ int owner(long long unit) const {
        const long long wide = (each + 1) * extra;
        return unit < wide ? (int)(unit / (each + 1)) : extra + (int)((unit - wide) / each);
    }
};

// A CTA's share: where it begins, and how many units it has.
struct Walk {
    long long unit, total, count, left;  // next unit, units of the call, of the share, of them still to do
    int list, tile, block;
};
// Consecutive units of one row tile.
struct Item {
    ListInfo li;
    long long unit;                      // the first one's number in the call
    int list, tile, b0, b1, blocks;      // key blocks b0 .. b1 - 1 of `blocks`
    bool first;                          // the CTA's first item
};
__device__ __forceinline__ bool next_item(const AttnArgs& a, Walk& w, int rows, int BK, Item& it) {
    if (w.left <= 0) return false;
    for (;;) {
        it.li = list_info(a, w.list, false);
        if (w.tile < tiles_of(it.li, a, rows)) break;
        ++w.list;
        w.tile = w.block = 0;
    }
    it.list = w.list;
    it.tile = w.tile;
    it.blocks = tile_blocks(it.li, a, w.tile, rows, BK);
    it.b0 = w.block;
    it.b1 = w.left < it.blocks - w.block ? w.block + (int)w.left : it.blocks;
    it.first = w.left == w.count;
    it.unit = w.unit;
    w.unit += it.b1 - it.b0;
    w.left -= it.b1 - it.b0;
    w.block = it.b1;
    if (w.block == it.blocks) {
        ++w.tile;
        w.block = 0;
    }
    return true;
}

__device__ __forceinline__ long long scan_up_ll(long long v, int d) { return __shfl_up_sync(0xffffffffu, v, d); }

// Where the CTA's share of the units begins.  Every thread calls it; *out (shared memory) is valid after the
// caller's next __syncthreads.  Reports lists that do not fit (CTA 0).
template <int THREADS>
__device__ void find_range(const AttnArgs& a, int BK, int rows, int cta, int ctas, Walk* out) {
    __shared__ long long warp_sum[THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (a.lists + THREADS - 1) / THREADS;
    const int r0 = min(a.lists, tid * per), r1 = min(a.lists, r0 + per);
    long long mine = 0;
    for (int r = r0; r < r1; ++r) {
        const ListInfo li = list_info(a, r, cta == 0);
        mine += list_units(li, a, rows, BK);
    }
    long long inc = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long x = scan_up_ll(inc, d);
        if (lane >= d) inc += x;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    long long before = 0, total = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w == warp) before = total;
        total += warp_sum[w];
    }
    long long at = before + inc - mine;
    const Division division(total, ctas);
    const long long first = division.begin(cta), end = division.begin(cta + 1);
    if (tid == 0) {
        out->unit = first;
        out->total = total;
        out->count = out->left = end - first;
        out->list = out->tile = out->block = 0;
    }
    __syncthreads();
    if (end > first && first >= at && first < at + mine) {
        for (int r = r0; r < r1; ++r) {
            const ListInfo li = list_info(a, r, false);
            const int tiles = tiles_of(li, a, rows);
            for (int t = 0; t < tiles; ++t) {
                const int nb = tile_blocks(li, a, t, rows, BK);
                if (first < at + nb) {
                    out->list = r;
                    out->tile = t;
                    out->block = (int)(first - at);
                    return;
                }
                at += nb;
            }
        }
    }
}

constexpr int kPagedMaxCtas = 160;             // grid of the persistent kernels, at most (one CTA per SM)
static_assert(2 * kPagedMaxCtas <= kCounters, "a counter per CTA and row tile");

// The CTAs that share a row tile: `parts` of them from c0 on.  Each leaves its part (maxima, sums, unnormalised output)
// in a slot of the workspace; few rows: the one that arrives last joins all, in the order of the keys; chunks: in pairs.  A CTA's first item
// is its slot 0, its last slot 1; only the tile's first CTA may have begun before the tile.  (Two tiles that are both
// shared begin in different CTAs, so c0 names the counter of the arrivals.)
struct Shared {
    int c0, parts, first_slot;
    __device__ __forceinline__ int slot(int p) const { return p == 0 ? first_slot : 2 * (c0 + p); }
};
__device__ __forceinline__ Shared shared_by(const Item& it, long long total, int ctas) {
    const Division d(total, ctas);
    const long long u0 = it.unit - it.b0;
    Shared s;
    s.c0 = d.owner(u0);
    s.parts = d.owner(u0 + it.blocks - 1) - s.c0 + 1;
    s.first_slot = 2 * s.c0 + (u0 > d.begin(s.c0) ? 1 : 0);
    return s;
}

// The pool as a rank-3 tensor (64 channels, rows of all pages, d / 64) in boxes of 64 channels x rows x chunks: a box lies in
// shared memory as [chunk][row][128 bytes], swizzled.
bool ea_paged_map(const ea_ctx* ctx, const ea_paged_shape& s, const void* pages, uint32_t rows, uint32_t chunks, CUtensorMap* map);
// Row tiles of 128 on the tensor cores (paged_chunk.cu).
size_t ea_paged_chunk_ws_floats(int d);
ea_status ea_launch_paged_chunk(const ea_ctx* ctx, const ea_paged_shape& s, const AttnArgs& a, const void* k_pages, const void* v_pages,
                                cudaStream_t st);

// ---- wrappers
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// m: maximum of the scores in units of log 2, l: sum of 2^(score - m)
__device__ __forceinline__ float lse_of(float m, float l) {
    return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}
// The scores' magnitude in units of log 2 from which on a row is refused: what a product's rounding leaves, 2^-24 of it, would be
// beyond what weights can hold (2^6 at this bound, the same in all weights of a row and in their sum).
constexpr float kFar = 1073741824.0f;
// The sum of a row that sees `seen` rows, or NaN (for its outputs too) where the largest of their scores is out of range.
__device__ __forceinline__ float sum_in_range(float m, float l, int seen) { return seen > 0 && !(fabsf(m) < kFar) ? NAN : l; }
// 1 / l for a row's normalisation: zero for a row that sees no key, NaN stays
__device__ __forceinline__ float inverse_sum(float l) { return l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l); }
__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&x)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(b0), "r"(b1));
}
