// The paged cache: pages taken and given back as lists grow and shrink, slot maps, and rows moved into and out
// of their slots.  (The attention that reads the cache is in paged_attn.cu.)
//
// A list is the cache of one (sequence, KV head).  With have = ceil(old / P) and want = ceil(new / P) pages of P
// rows, the lists that grow take N = sum max(0, want - have) pages, those that shrink give M back.  Both sides are
// numbered, takes in ascending order of (list, page), releases in descending order, and item t < max(N, M) is one
// page that changes hands:
//     page(t)  = t < M ? the t-th released page : free[top - 1 - (t - M)]
//     t < N    : page(t) becomes the table entry of the t-th take
//     N <= t   : page(t) is pushed, free[top + t - N]
// So the free list is either only read or only written, every entry of the table has one writer, and no order
// between threads matters.  A shrink that undoes a growth leaves the free list as it was.
#include "paged.h"
#include "fast_div.cuh"
#include "ptx_sm100.cuh"

namespace {

// Four paths, times on the device for a plan that grows lists and one that takes the pages back, in a CUDA graph:
//  * a plan with a slot map of at most kClusterSlots slots: one cluster, one launch.  8 lists x 64 rows 10.0 us, 65 536 slots
//    13.3 (13.6 with three launches); beyond, the slots want all SMs: 131 072 slots 15.1 us against 13.5, 288 000 27.9
//    against 19.0.  (A single CTA, without cluster barriers, is no faster for small plans: 10.2 us at 512 slots, 12.7
//    against 10.5 at 8192.)
//  * a plan without a slot map: one launch over all SMs, as nothing bounds the pages that move but the pool (384 lists
//    of up to 16 384 rows, a growth with its slots and this undoing: 30 us, 38 with the undoing in a cluster)
//  * a slot map of standing tables: one launch over all SMs (288 lists of up to 8192 rows: 9 us with the launch)
//  * more lists than a CTA keeps prefixes of: scan, pages and slots in three launches
constexpr int kSelfScanLists = 4096;      // up to here every CTA scans the lengths itself (48 KiB of prefixes)
constexpr int kScanSmem = 3 * (kSelfScanLists + 1) * 4;
constexpr int kClusterSlots = 65536, kPlanCluster = 8;
constexpr int kScanThreads = 1024, kMoveThreads = 256;

struct PlanArgs {
    const int32_t* old_lens;     // first rows (slots only)
    const int32_t* new_lens;     // end rows
    int32_t* table;
    int32_t* free_pages;         // nullptr: the tables stand (ea_page_slots)
    int32_t* n_free;
    int32_t* slots;
    int32_t* offsets;
    int32_t* scratch;            // prefixes of more than kSelfScanLists lists, and the totals
    unsigned* counter;           // arrivals of page_resize_kernel, zero between calls
    unsigned* operand;           // the scratch lies where a fused statistics operand would
    int* status;                 // [1]: page status word
    int lists, Hkv, shift, n_pages, max_pages, by_token, slot_capacity;
    FastDiv div_hkv;             // by Hkv
};

// What a scan finds.  All-or-nothing: a call that cannot be served has n_take = n_give = rows = 0.
struct Totals {
    int n_take, n_give, rows, top, bad;
};

__device__ __forceinline__ int pages_of(int rows, int shift) { return (int)(((unsigned)rows + (1u << shift) - 1u) >> shift); }

struct Tally {
    long long take, give, rows;
    int bad;
};

__device__ __forceinline__ void count_list(const PlanArgs& a, int r, Tally& t) {
    const int o = a.old_lens[r], n = a.new_lens[r];
    const long long cap = (long long)a.max_pages << a.shift;
    if (o < 0 || n < 0 || o > cap || n > cap) {
        t.bad = 1;
        return;
    }
    const int have = pages_of(o, a.shift), want = pages_of(n, a.shift);
    t.take += want > have ? want - have : 0;
    t.give += have > want ? have - want : 0;
    t.rows += n > o ? n - o : 0;
    // token order puts the heads of a token side by side: they must gain the same rows
    const int head0 = quotient(r, a.div_hkv) * a.Hkv;
    if (a.by_token && r != head0) {
        const int o0 = a.old_lens[head0], n0 = a.new_lens[head0];
        if ((n > o ? n - o : 0) != (n0 > o0 ? n0 - o0 : 0)) t.bad = 1;
    }
}

// Exclusive prefixes of pages taken, pages given back and rows gained, over all lists, into take / give / rows
// (lists + 1 entries each; shared or global memory).  Every thread of the CTA calls it; the totals are returned
// to all of them.  Entries hold 32 bits: totals beyond that are refused.
template <int THREADS>
__device__ Totals scan_lists(const PlanArgs& a, int32_t* take, int32_t* give, int32_t* rows) {
    constexpr int WARPS = THREADS / 32;
    __shared__ long long sums[3][WARPS];
    __shared__ Totals total;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (a.lists + THREADS - 1) / THREADS;
    const int r0 = min(a.lists, tid * per), r1 = min(a.lists, r0 + per);
    Tally mine = {0, 0, 0, 0};
    for (int r = r0; r < r1; ++r) count_list(a, r, mine);
    auto scan = [&](long long v) {                       // inclusive, over a warp
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += x;
        }
        return v;
    };
    const long long it = scan(mine.take), ig = scan(mine.give), ir = scan(mine.rows);
    if (lane == 31) {
        sums[0][warp] = it;
        sums[1][warp] = ig;
        sums[2][warp] = ir;
    }
    int bad = __syncthreads_or(mine.bad);
    // every warp scans the warps' sums
    long long before[3], all[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const long long own = lane < WARPS ? sums[k][lane] : 0, inc = scan(own);
        before[k] = __shfl_sync(0xffffffffu, inc - own, warp);
        all[k] = __shfl_sync(0xffffffffu, inc, 31);
    }
    if (tid == 0) {
        int top = 0;
        if (a.free_pages) {
            top = *a.n_free;
            if (top < 0 || top > a.n_pages || all[0] - all[1] > top || top + all[1] - all[0] > a.n_pages || all[0] > a.n_pages || all[1] > a.n_pages)
                bad = 1;
        }
        if (all[2] > 0x7fffffffLL) bad = 1;
        if (a.slots && all[2] > a.slot_capacity) bad = 1;
        total = bad ? Totals{0, 0, 0, top, 1} : Totals{(int)all[0], (int)all[1], (int)all[2], top, 0};
    }
    __syncthreads();
    const Totals out = total;
    Tally at = {before[0] + it - mine.take, before[1] + ig - mine.give, before[2] + ir - mine.rows, 0};
    for (int r = r0; r < r1; ++r) {
        take[r] = out.bad ? 0 : (int)at.take;
        give[r] = out.bad ? 0 : (int)at.give;
        rows[r] = out.bad ? 0 : (int)at.rows;
        if (r + 1 < r1) count_list(a, r, at);
    }
    if (tid == 0) {
        take[a.lists] = out.n_take;
        give[a.lists] = out.n_give;
        rows[a.lists] = out.rows;
    }
    __syncthreads();
    return out;
}

// last r with prefix[r] <= x (x < prefix[lists])
__device__ __forceinline__ int find_list(const int32_t* prefix, int lists, int x) {
    int lo = 0, hi = lists;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Items t0, t0 + step, ... of the pages that change hands.
__device__ void move_pages(const PlanArgs& a, const Totals& tot, const int32_t* take, const int32_t* give, int t0, int step) {
    const int items = max(tot.n_take, tot.n_give);
    for (int t = t0; t < items; t += step) {
        int page;
        if (t < tot.n_give) {
            const int x = tot.n_give - 1 - t;                       // last list first, last page first
            const int r = find_list(give, a.lists, x);
            int32_t* entry = a.table + (size_t)r * a.max_pages + pages_of(a.new_lens[r], a.shift) + (x - give[r]);
            page = *entry;
            *entry = -1;
        } else {
            page = a.free_pages[tot.top - 1 - (t - tot.n_give)];
        }
        if ((unsigned)page >= (unsigned)a.n_pages) a.status[1] = (int)EA_ERR_PAGES;     // the caller's table or free list is wrong
        if (t < tot.n_take) {
            const int r = find_list(take, a.lists, t);
            a.table[(size_t)r * a.max_pages + pages_of(a.old_lens[r], a.shift) + (t - take[r])] = page;
        } else {
            a.free_pages[tot.top + t - tot.n_take] = page;
        }
    }
}

__device__ __forceinline__ int slot_of(const PlanArgs& a, int r, int p) {
    const int page = a.table[(size_t)r * a.max_pages + (p >> a.shift)];
    return (unsigned)page < (unsigned)a.n_pages ? (page << a.shift) + (p & ((1 << a.shift) - 1)) : -1;
}

// The slot of new row t of the call (rows old .. new of every list), -1 behind the last.  `r`, `next`: in list order, the
// list of the thread's slot before and where it ends.
__device__ __forceinline__ int slot_at(const PlanArgs& a, const Totals& tot, const int32_t* rows, long long t, int& r, int& next) {
    if (t >= tot.rows) return -1;
    if (a.by_token) {
        // rows[] counts Hkv rows per token: token t / Hkv begins its sequence at rows[s * Hkv] / Hkv
        const int token = quotient((int)t, a.div_hkv), g = (int)t - token * a.Hkv;
        const int s = quotient(find_list(rows, a.lists, token * a.Hkv), a.div_hkv);      // lists of a sequence gain alike
        const int list = s * a.Hkv + g;
        return slot_of(a, list, a.old_lens[list] + token - quotient(rows[s * a.Hkv], a.div_hkv));
    }
    if (r < 0 || t >= next) {
        r = find_list(rows, a.lists, (int)t);
        next = rows[r + 1];
    }
    return slot_of(a, r, a.old_lens[r] + (int)t - rows[r]);
}

// The CTA's share of the slots, side by side, so that a thread mostly stays in the list of its slot before: one at a time
// where they are few (the chain of dependent loads is the time), four where they are many.
__device__ void write_slots(const PlanArgs& a, const Totals& tot, const int32_t* rows) {
    int r = -1, next = 0;
    const bool wide = a.slot_capacity > (long long)gridDim.x * blockDim.x && (reinterpret_cast<uintptr_t>(a.slots) & 15u) == 0;
    const long long quads = wide ? a.slot_capacity / 4 : 0;
    const long long share = (quads + gridDim.x - 1) / gridDim.x, end = min(quads, (blockIdx.x + 1) * share);
    for (long long q = blockIdx.x * share + threadIdx.x; q < end; q += blockDim.x) {
        int v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = slot_at(a, tot, rows, q * 4 + e, r, next);
        reinterpret_cast<int4*>(a.slots)[q] = make_int4(v[0], v[1], v[2], v[3]);
    }
    r = -1;
    for (long long t = quads * 4 + (long long)blockIdx.x * blockDim.x + threadIdx.x; t < a.slot_capacity; t += (long long)gridDim.x * blockDim.x)
        a.slots[t] = slot_at(a, tot, rows, t, r, next);
}

// Offsets (list order: lists + 1 row offsets; token order: sequences + 1 token offsets), the free count, the status.
__device__ void write_offsets(const PlanArgs& a, const Totals& tot, const int32_t* rows) {
    if (a.offsets) {
        const int n = a.by_token ? a.lists / a.Hkv : a.lists;
        for (int i = threadIdx.x; i <= n; i += blockDim.x) a.offsets[i] = a.by_token ? quotient(rows[i * a.Hkv], a.div_hkv) : rows[i];
    }
    if (threadIdx.x == 0) {
        if (a.free_pages && !tot.bad) *a.n_free = tot.top - tot.n_take + tot.n_give;
        if (tot.bad) a.status[1] = (int)EA_ERR_PAGES;
    }
}

// The whole plan in one cluster (one launch): for a generation step further launches would cost more than the work.
// Every CTA scans the lengths for itself; the free count is read before the first cluster barrier and written after
// the last.
__global__ void __launch_bounds__(kScanThreads) page_plan_cluster_kernel(const PlanArgs a) {
    extern __shared__ int32_t prefix[];
    int32_t *take = prefix, *give = take + a.lists + 1, *rows = give + a.lists + 1;
    const Totals tot = scan_lists<kScanThreads>(a, take, give, rows);
    const int t0 = blockIdx.x * kScanThreads + threadIdx.x, step = gridDim.x * kScanThreads;
    ptx::cluster_sync();
    if (a.free_pages) {
        move_pages(a, tot, take, give, t0, step);
        ptx::cluster_sync();                                        // the slots read the entries just written
    }
    if (a.slots) write_slots(a, tot, rows);
    if (blockIdx.x == 0) write_offsets(a, tot, rows);
}

// A plan without slots over all SMs in one launch: every CTA scans the lengths for itself and moves its share of the
// pages; the free count is written by the CTA that arrives last, when all others have read it.
__global__ void __launch_bounds__(kMoveThreads) page_resize_kernel(const PlanArgs a) {
    extern __shared__ int32_t prefix[];
    __shared__ bool last;
    int32_t *take = prefix, *give = take + a.lists + 1, *rows = give + a.lists + 1;
    const Totals tot = scan_lists<kMoveThreads>(a, take, give, rows);
    move_pages(a, tot, take, give, blockIdx.x * kMoveThreads + threadIdx.x, gridDim.x * kMoveThreads);
    __syncthreads();
    if (threadIdx.x == 0) last = arrives_last(a.counter, gridDim.x);
    __syncthreads();
    if (last) write_offsets(a, tot, rows);
}

// Larger plans: prefixes and totals into the workspace, then the pages, then the slots.
__global__ void __launch_bounds__(kScanThreads) page_scan_kernel(const PlanArgs a) {
    int32_t *take = a.scratch, *give = take + a.lists + 1, *rows = give + a.lists + 1;
    const Totals tot = scan_lists<kScanThreads>(a, take, give, rows);
    if (threadIdx.x == 0) {
        *reinterpret_cast<Totals*>(rows + a.lists + 1) = tot;
        *a.operand = 0;
    }
    write_offsets(a, tot, rows);
}

__global__ void __launch_bounds__(kMoveThreads) page_move_kernel(const PlanArgs a) {
    const int32_t *take = a.scratch, *give = take + a.lists + 1;
    const Totals tot = *reinterpret_cast<const Totals*>(give + 2 * (a.lists + 1));
    move_pages(a, tot, take, give, blockIdx.x * kMoveThreads + threadIdx.x, gridDim.x * kMoveThreads);
}

// SCAN: the tables stand and the lists are few: every CTA scans the lengths for itself, and one launch is all.
template <bool SCAN>
__global__ void __launch_bounds__(kMoveThreads) page_slots_kernel(const PlanArgs a) {
    extern __shared__ int32_t prefix[];
    const int32_t* rows;
    Totals tot;
    if (SCAN) {
        rows = prefix + 2 * (a.lists + 1);
        tot = scan_lists<kMoveThreads>(a, prefix, prefix + a.lists + 1, prefix + 2 * (a.lists + 1));
        if (blockIdx.x == 0) write_offsets(a, tot, rows);
    } else {
        rows = a.scratch + 2 * (a.lists + 1);
        tot = *reinterpret_cast<const Totals*>(rows + a.lists + 1);
    }
    if (a.slots) write_slots(a, tot, rows);
}

// rows <-> slots, 16 bytes of K and of V per thread and step.  A slot of -1 names no row; any other number outside the
// pool is reported and skipped.  src: row i of the rows side begins at (i / group) * group_stride + (i % group) * d
// elements (dense rows: group = 1, group_stride = d).  HBM: 342 MB of compacted rows into their slots 116 us, 0.91 of the
// measured copy rate; the rows of one token of one layer 1.9 us with the launch.
template <bool STORE, int LPR /* 16-byte pieces per row */>
__global__ void __launch_bounds__(256) page_rows_kernel(const int32_t* __restrict__ slots, long long n_rows, uint4* __restrict__ k_rows,
                                                        uint4* __restrict__ v_rows, int group, long long k_stride, long long v_stride,
                                                        uint4* __restrict__ k_pages, uint4* __restrict__ v_pages, int n_slots, int* status) {
    constexpr int U = 4;                       // rows in flight per thread: eight 16-byte loads hide the latency
    constexpr int ROWS = 256 / LPR;            // rows of one step of the CTA
    const int piece = threadIdx.x % LPR;
    const long long step = (long long)gridDim.x * ROWS * U;
    for (long long r0 = (long long)blockIdx.x * ROWS * U + threadIdx.x / LPR; r0 < n_rows; r0 += step) {
        uint4 k[U], v[U];
        int slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * ROWS;
            slot[u] = r < n_rows ? __ldg(slots + r) : -1;
            if (slot[u] >= n_slots || slot[u] < -1) {
                status[1] = (int)EA_ERR_PAGES;
                slot[u] = -1;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * ROWS;
            if (slot[u] < 0) continue;
            if (STORE) {
                const long long gi = group == 1 ? r : r / group, ge = group == 1 ? 0 : (r % group) * LPR;
                k[u] = __ldcs(k_rows + gi * k_stride + ge + piece);
                v[u] = __ldcs(v_rows + gi * v_stride + ge + piece);
            } else {
                k[u] = __ldcs(k_pages + (long long)slot[u] * LPR + piece);
                v[u] = __ldcs(v_pages + (long long)slot[u] * LPR + piece);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * ROWS;
            if (slot[u] < 0) continue;
            if (STORE) {
                k_pages[(long long)slot[u] * LPR + piece] = k[u];
                v_pages[(long long)slot[u] * LPR + piece] = v[u];
            } else {
                k_rows[r * LPR + piece] = k[u];
                v_rows[r * LPR + piece] = v[u];
            }
        }
    }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

size_t scan_bytes(const ea_paged_shape& s) { return (3 * ((size_t)s.n_seqs * s.n_kv_heads + 1) + sizeof(Totals) / 4) * 4; }

// Lists up to kSelfScanLists need no scratch when one launch does it all, but whether it does depends on the call.
ea_status launch_plan(const ea_ctx* ctx, PlanArgs a, cudaStream_t st) {
    const int smem = 3 * (a.lists + 1) * 4;
    const bool few = a.lists <= kSelfScanLists;
    const bool resize = a.free_pages != nullptr;
    const long long quads = ((long long)a.slot_capacity + 3) / 4;
    const long long want = (quads + kMoveThreads - 1) / kMoveThreads, cap = (long long)ctx->sm_count * 4;
    const unsigned slot_grid = (unsigned)(want < 1 ? 1 : want < cap ? want : cap);
    if (few && !resize) {
        static std::atomic<uint64_t> done{0};
        const ea_status err = ea_allow_smem(page_slots_kernel<true>, kScanSmem, ctx->device, done);
        if (err != EA_OK) return err;
        page_slots_kernel<true><<<slot_grid, kMoveThreads, smem, st>>>(a);
        ea_count_launches(ctx, 1);
        return EA_CHECK_LAUNCH();
    }
    if (few && a.slot_capacity == 0) {
        // nothing bounds the pages that move but the pool
        static std::atomic<uint64_t> done{0};
        const ea_status err = ea_allow_smem(page_resize_kernel, kScanSmem, ctx->device, done);
        if (err != EA_OK) return err;
        const long long ctas = ((long long)a.n_pages + 4 * kMoveThreads - 1) / (4 * kMoveThreads), most = ctx->sm_count;
        page_resize_kernel<<<(unsigned)(ctas < 1 ? 1 : ctas < most ? ctas : most), kMoveThreads, smem, st>>>(a);
        ea_count_launches(ctx, 1);
        return EA_CHECK_LAUNCH();
    }
    if (few && a.slot_capacity <= kClusterSlots) {
        static std::atomic<uint64_t> done{0};
        const ea_status err = ea_allow_smem(page_plan_cluster_kernel, kScanSmem, ctx->device, done);
        if (err != EA_OK) return err;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(kPlanCluster);
        cfg.blockDim = dim3(kScanThreads);
        cfg.dynamicSmemBytes = (size_t)smem;
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kPlanCluster;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        EA_CUDA_TRY(cudaLaunchKernelEx(&cfg, page_plan_cluster_kernel, a));
        ea_count_launches(ctx, 1);
        return EA_CHECK_LAUNCH();
    }
    page_scan_kernel<<<1, kScanThreads, 0, st>>>(a);
    if (resize) {
        const long long pages = (a.n_pages + kMoveThreads - 1) / kMoveThreads, most = (long long)ctx->sm_count * 4;
        page_move_kernel<<<(unsigned)(pages < 1 ? 1 : pages < most ? pages : most), kMoveThreads, 0, st>>>(a);
    }
    if (a.slot_capacity > 0) page_slots_kernel<false><<<slot_grid, kMoveThreads, 0, st>>>(a);
    ea_count_launches(ctx, 1 + (resize ? 1 : 0) + (a.slot_capacity > 0 ? 1 : 0));
    return EA_CHECK_LAUNCH();
}

ea_status plan_call(ea_ctx* ctx, const ea_paged_shape* shape, const int32_t* old_lens, const int32_t* new_lens, int32_t* table,
                    int32_t* free_pages, int32_t* n_free, bool resize, int32_t order, int32_t* slots, int32_t slot_capacity,
                    int32_t* offsets, void* cuda_stream) {
    if (!ctx) return EA_ERR_INVALID_ARG;
    ea_status st = ea_check_paged_shape(shape);
    if (st != EA_OK) return st;
    if (order != EA_SLOTS_BY_LIST && order != EA_SLOTS_BY_TOKEN) return EA_ERR_INVALID_ARG;
    if (slot_capacity < 0 || (slot_capacity > 0 && !slots)) return EA_ERR_INVALID_ARG;
    const long long lists = (long long)shape->n_seqs * shape->n_kv_heads;
    if (lists > 0 && (!old_lens || !new_lens || (shape->max_pages > 0 && !table))) return EA_ERR_INVALID_ARG;
    if (resize && (!n_free || (shape->n_pages > 0 && !free_pages))) return EA_ERR_INVALID_ARG;
    if (!aligned4(old_lens) || !aligned4(new_lens) || !aligned4(table) || !aligned4(free_pages) || !aligned4(n_free) ||
        !aligned4(slots) || !aligned4(offsets))
        return EA_ERR_INVALID_ARG;
    if (ctx->workspace_bytes < scan_bytes(*shape)) return EA_ERR_WORKSPACE;
    if (lists == 0 && slot_capacity == 0 && !offsets) return EA_OK;
    const long long i32 = sizeof(int32_t);
    const Span spans[] = {{old_lens, lists * i32, false}, {new_lens, lists * i32, false},
                          {table, lists * shape->max_pages * i32, resize}, {free_pages, resize ? shape->n_pages * i32 : 0, true},
                          {n_free, resize ? i32 : 0, true}, {slots, slot_capacity * i32, true},
                          {offsets, (order == EA_SLOTS_BY_TOKEN ? shape->n_seqs + 1LL : lists + 1) * i32, true}};
    if (outputs_overlap(spans)) return EA_ERR_INVALID_ARG;
    PlanArgs a = {};
    a.old_lens = old_lens;
    a.new_lens = new_lens;
    a.table = table;
    a.free_pages = resize ? (free_pages ? free_pages : n_free) : nullptr;      // an empty pool is never indexed
    a.n_free = n_free;
    a.slots = slots;
    a.offsets = offsets;
    a.scratch = static_cast<int32_t*>(ctx->workspace);
    a.status = ctx->status_dev;
    a.counter = ctx->counters + kCounters - 1;
    a.operand = ea_operand_word(ctx);
    a.lists = (int)lists;
    a.Hkv = shape->n_kv_heads;
    a.div_hkv = fast_div(a.Hkv);
    a.shift = __builtin_ctz((unsigned)shape->page_rows);
    a.n_pages = shape->n_pages;
    a.max_pages = shape->max_pages;
    a.by_token = order == EA_SLOTS_BY_TOKEN;
    a.slot_capacity = slot_capacity;
    int prev = 0;
    EA_CUDA_TRY(cudaGetDevice(&prev));
    if (prev != ctx->device) EA_CUDA_TRY(cudaSetDevice(ctx->device));
    ctx->image_ready = false;                       // the scratch lies where fused statistics keep their images
    st = launch_plan(ctx, a, static_cast<cudaStream_t>(cuda_stream));
    if (prev != ctx->device) cudaSetDevice(prev);
    return st;
}

template <bool STORE>
ea_status rows_call(ea_ctx* ctx, const ea_paged_shape* shape, const int32_t* slots, int64_t n_rows, void* k_rows, void* v_rows,
                    int64_t k_stride, int64_t v_stride, void* k_pages, void* v_pages, void* cuda_stream) {
    if (!ctx) return EA_ERR_INVALID_ARG;
    ea_status st = ea_check_paged_shape(shape);
    if (st != EA_OK) return st;
    if (n_rows < 0 || n_rows > 0x7fffffffLL) return EA_ERR_INVALID_ARG;
    const int d = shape->head_dim, lpr = d / 8;
    const int64_t dense = (int64_t)shape->n_kv_heads * d;
    const bool strided = STORE && (k_stride != 0 || v_stride != 0);
    if (STORE) {
        // strides: elements between groups of n_kv_heads rows (the tokens of a fused projection), 0 = dense
        if (k_stride < 0 || v_stride < 0 || k_stride % 8 != 0 || v_stride % 8 != 0) return EA_ERR_INVALID_ARG;
        if ((k_stride != 0 && k_stride < dense) || (v_stride != 0 && v_stride < dense)) return EA_ERR_INVALID_ARG;
        if (strided && n_rows % shape->n_kv_heads != 0) return EA_ERR_INVALID_ARG;
    }
    if (n_rows == 0) return EA_OK;
    if (!slots || !k_rows || !v_rows || (shape->n_pages > 0 && (!k_pages || !v_pages))) return EA_ERR_INVALID_ARG;
    if (!aligned4(slots) || !aligned16(k_rows) || !aligned16(v_rows) || !aligned16(k_pages) || !aligned16(v_pages)) return EA_ERR_INVALID_ARG;
    const long long groups = n_rows / shape->n_kv_heads, pool = (long long)shape->n_pages * shape->page_rows * d * 2;
    auto rows_bytes = [&](int64_t stride) { return 2 * (strided && stride ? (groups - 1) * stride + dense : n_rows * d); };
    const Span spans[] = {{slots, n_rows * 4, false}, {k_rows, rows_bytes(k_stride), !STORE}, {v_rows, rows_bytes(v_stride), !STORE},
                          {k_pages, pool, STORE}, {v_pages, pool, STORE}};
    if (outputs_overlap(spans)) return EA_ERR_INVALID_ARG;
    int prev = 0;
    EA_CUDA_TRY(cudaGetDevice(&prev));
    if (prev != ctx->device) EA_CUDA_TRY(cudaSetDevice(ctx->device));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int group = strided ? shape->n_kv_heads : 1;
    const long long ks = strided ? (k_stride ? k_stride : dense) / 8 : lpr, vs = strided ? (v_stride ? v_stride : dense) / 8 : lpr;
    const long long per = 256 / lpr * 4, want = (n_rows + per - 1) / per, cap = (long long)ctx->sm_count * 8;
    const unsigned grid = (unsigned)(want < cap ? want : cap);
    const int n_slots = shape->n_pages * shape->page_rows;
    auto kernel = lpr == 8 ? page_rows_kernel<STORE, 8> : lpr == 16 ? page_rows_kernel<STORE, 16> : page_rows_kernel<STORE, 32>;
    kernel<<<grid, 256, 0, stream>>>(slots, n_rows, static_cast<uint4*>(k_rows), static_cast<uint4*>(v_rows), group, ks, vs,
                                     static_cast<uint4*>(k_pages), static_cast<uint4*>(v_pages), n_slots, ctx->status_dev);
    ea_count_launches(ctx, 1);
    st = EA_CHECK_LAUNCH();
    if (prev != ctx->device) cudaSetDevice(prev);
    return st;
}

}  // namespace

ea_status ea_check_paged_shape(const ea_paged_shape* s) {
    if (!s) return EA_ERR_INVALID_ARG;
    if (s->n_seqs < 0 || s->n_q_heads < 1 || s->n_kv_heads < 1 || s->n_pages < 0 || s->max_pages < 0) return EA_ERR_INVALID_ARG;
    if (s->n_q_heads % s->n_kv_heads != 0) return EA_ERR_INVALID_ARG;
    if (s->head_dim != 64 && s->head_dim != 128 && s->head_dim != 256) return EA_ERR_UNSUPPORTED;
    if (s->page_rows != 16 && s->page_rows != 32 && s->page_rows != 64 && s->page_rows != 128) return EA_ERR_UNSUPPORTED;
    if ((long long)s->n_seqs * s->n_kv_heads > 65535LL) return EA_ERR_UNSUPPORTED;
    // slot numbers and list lengths are 32-bit
    if ((long long)s->n_pages * s->page_rows > 0x7fffffffLL || (long long)s->max_pages * s->page_rows > (1LL << 30)) return EA_ERR_UNSUPPORTED;
    return EA_OK;
}

extern "C" {

ea_status ea_paged_workspace_bytes(const ea_paged_shape* shape, int32_t max_q, size_t* out_bytes) {
    if (!out_bytes || max_q < 0) return EA_ERR_INVALID_ARG;
    ea_status st = ea_check_paged_shape(shape);
    if (st != EA_OK) return st;
    const size_t scan = scan_bytes(*shape), attn = ea_paged_attn_ws_bytes(*shape, max_q);
    *out_bytes = ea_align_up(scan > attn ? scan : attn, 256);
    return EA_OK;
}

ea_status ea_page_plan(ea_ctx* ctx, const ea_paged_shape* shape, const int32_t* old_lens, const int32_t* new_lens,
                       int32_t* block_table, int32_t* free_pages, int32_t* n_free, int32_t order, int32_t* slots_opt,
                       int32_t slot_capacity, int32_t* offsets_opt, void* cuda_stream) {
    return plan_call(ctx, shape, old_lens, new_lens, block_table, free_pages, n_free, true, order, slots_opt, slot_capacity,
                     offsets_opt, cuda_stream);
}

ea_status ea_page_slots(ea_ctx* ctx, const ea_paged_shape* shape, const int32_t* block_table, const int32_t* first_row,
                        const int32_t* end_row, int32_t order, int32_t* slots, int32_t slot_capacity, int32_t* offsets_opt,
                        void* cuda_stream) {
    return plan_call(ctx, shape, first_row, end_row, const_cast<int32_t*>(block_table), nullptr, nullptr, false, order, slots,
                     slot_capacity, offsets_opt, cuda_stream);
}

ea_status ea_page_store(ea_ctx* ctx, const ea_paged_shape* shape, const int32_t* slots, int64_t n_rows, const void* k_new,
                        const void* v_new, int64_t k_stride, int64_t v_stride, void* k_pages, void* v_pages, void* cuda_stream) {
    return rows_call<true>(ctx, shape, slots, n_rows, const_cast<void*>(k_new), const_cast<void*>(v_new), k_stride, v_stride,
                           k_pages, v_pages, cuda_stream);
}

ea_status ea_page_load(ea_ctx* ctx, const ea_paged_shape* shape, const int32_t* slots, int64_t n_rows, const void* k_pages,
                       const void* v_pages, void* k_out, void* v_out, void* cuda_stream) {
    return rows_call<false>(ctx, shape, slots, n_rows, k_out, v_out, 0, 0, const_cast<void*>(k_pages), const_cast<void*>(v_pages),
                            cuda_stream);
}

}  // extern "C"
