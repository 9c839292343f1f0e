// Attention over the paged key/value cache, prefixes shared by a group of sequences read once for all of them.
//
//   out = sum_j p_j v_j / l,  p_j = exp2(c (s_j - m)),  s_j = q . k_j,  c = scale log2(e),  l = sum_j p_j,
// for any m; m follows the running maximum, so that the sums over ranges of keys can be joined:
//   (m, l, o), (m', l', o') -> M = max(m, m'), l 2^(c (m - M)) + l' 2^(c (m' - M)), o likewise.
//
// The rows of an item are all (query token, query head) pairs that read the same kv head of the same pages: the
// tokens of one sequence times the heads of its group, or those of all sequences that share a prefix.  Rows of a
// shared prefix thus meet its keys once, as the rows of one matrix product, and their other keys in items of their own.
//
// k_attend: one block per SM.  The tiles (128 keys) of all items and heads lie on one line; every block takes an
// equal stretch of it, so work is even whatever the lengths, and an item is split where two stretches meet.  A warp brings tiles
// by TMA (a box per page: keys of a page and head are contiguous; a page number past the pool gives zeros), a
// thread issues tcgen05.mma, two groups of four warps do the softmax:
//   S = Q K^T    128 x 128 x D, both from shared memory, into TMEM;
//   P = exp2(..) one TMEM lane (row) per thread, so no value crosses threads; P overwrites S in TMEM, 16 bits;
//   O += P V     128 x D x 128, P from TMEM, V from shared memory as it lies (the N dimension contiguous).
// With more than 128 rows the two groups hold the two halves of the rows and share every tile, else they take
// tiles in turn; with at most 64 (32) rows the rows lie in TMEM twice (four times), each copy with its own half
// (quarter) of a tile's keys, so that all four warps work on few rows.  O is rescaled only when a row's
// maximum has grown by more than 2^8: until then P stays below 2^8 and nothing is lost in 32-bit sums.
#include <cuda.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "sim.h"
#include "sim_kv_internal.h"

namespace simgb {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int kPlan = 1024;
constexpr int kStage = 128 * 17;       // floats through which a group's results pass
constexpr int kSegs = 4;               // segments that the loading warp may be ahead
constexpr int kShareCost = 4;          // tiles of 128 rows that a second partial result of as many rows costs
constexpr float kGrow = 8.f;           // log2 of what P may reach before O is rescaled

// Tiles [line_at(c), line_at(c + 1)) of a list's line are block c's.
__device__ __forceinline__ int64_t line_at(int64_t units, int c, int blocks) { return units * c / blocks; }
__device__ __forceinline__ int block_at(int64_t units, int64_t u, int blocks) { return int(((u + 1) * blocks - 1) / units); }

// ---- plan ---------------------------------------------------------------------------------------------------

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Entry i's query tokens [a, a + t), none if the offsets are not in order; the table's row, or -1 (and no keys).
struct Entry {
    int a, t, seq, len;
};
__device__ __forceinline__ Entry entry_at(const sim_kv &kv, const sim_kv_batch &b, int i) {
    Entry e;
    e.a = b.cu_q[i];
    const int z = b.cu_q[i + 1], s = b.seqs[i];
    const bool ok = 0 <= e.a && e.a <= z && z <= b.n_q;
    e.t = ok ? z - e.a : 0;
    e.seq = unsigned(s) < unsigned(kv.max_seqs) ? s : -1;
    e.len = e.seq >= 0 ? min(kv.length[s], kv.max_pages * kv.page_size) : 0;
    return e;
}

// Group of entry i (the last that begins at or before it), -1 without groups.
__device__ __forceinline__ int group_of(const sim_kv_batch &b, int i) {
    int lo = -1, hi = b.n_groups;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (b.cu_group[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo >= 0 && i < b.cu_group[lo + 1] ? lo : -1;
}

// A warp for each entry: the pages that its table begins with like that of its group's first entry, all of whose
// keys each of its queries sees.
__global__ void __launch_bounds__(256) k_plan_shared(const sim_kv kv, const sim_kv_batch b) {
    kv_wait_previous();
    const KvPlan p = kv_plan(kv, b);
    const int i = (blockIdx.x * 256 + threadIdx.x) >> 5, lane = threadIdx.x & 31;
    if (i >= b.n) return;
    const int g = group_of(b, i);
    const Entry e = entry_at(kv, b, i);
    if (g < 0 || e.t == 0) {
        if (lane == 0) p.same[i] = INT_MAX;
        return;
    }
    const int first = max(b.cu_group[g], 0), s0 = b.seqs[first];
    int same = 0;
    if (unsigned(s0) < unsigned(kv.max_seqs)) {
        const int most = min(max(e.len - e.t + 1, 0), kv.length[s0]) / kv.page_size;
        const int32_t *x = kv.table + int64_t(e.seq) * kv.max_pages, *y = kv.table + int64_t(s0) * kv.max_pages;
        same = most;
        for (int j0 = 0; j0 < most; j0 += 128) {
            bool differ[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int j = j0 + 32 * k + lane;
                differ[k] = j < most && x[j] != y[j];
            }
            int at = INT_MAX;
#pragma unroll
            for (int k = 3; k >= 0; --k) {
                const unsigned m = __ballot_sync(FULL, differ[k]);
                if (m) at = j0 + 32 * k + __ffs(m) - 1;
            }
            if (at != INT_MAX) {
                same = at;
                break;
            }
        }
    }
    if (lane == 0) p.same[i] = same;
}

__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t *sums, int64_t &total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t y = __shfl_up_sync(FULL, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) sums[w] = x;
    __syncthreads();
    if (w == 0) {
        int64_t s = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t y = __shfl_up_sync(FULL, s, d);
            if (lane >= d) s += y;
        }
        sums[lane] = s;
    }
    __syncthreads();
    total = sums[31];
    const int64_t before = (w ? sums[w - 1] : 0) + x - v;
    __syncthreads();
    return before;
}

// Tile rows of 128 that r query rows take: two where they are more than 128 in their block of 256.
__device__ __forceinline__ int tile_rows(int r) {
    const int rem = r % kAttRows;
    return 2 * (r / kAttRows) + (rem > kAttRows / 2 ? 2 : rem > 0);
}
__device__ __forceinline__ int heavy_items(int r) { return r / kAttRows + (r % kAttRows > kAttRows / 2); }
__device__ __forceinline__ int light_items(int r) { return r % kAttRows > 0 && r % kAttRows <= kAttRows / 2; }

// One block: which prefixes are shared, the items of every source (a group's prefix, an entry's own keys), and
// where each begins on its list's line of work.
__global__ void __launch_bounds__(kPlan) k_plan_items(const sim_kv kv, const sim_kv_batch b, int sms) {
    __shared__ int64_t sums[32];
    kv_wait_previous();
    const KvPlan p = kv_plan(kv, b);
    const int tid = threadIdx.x, ng = b.n_groups, n_src = ng + b.n, G = b.q_heads / kv.n_kv_heads, P = kv.page_size;
    // Offsets that are not in order: no queries at all, or no groups.
    bool order = true, groups = true, known = true;
    for (int i = tid; i < b.n; i += kPlan) {
        order = order && 0 <= b.cu_q[i] && b.cu_q[i] <= b.cu_q[i + 1] && b.cu_q[i + 1] <= b.n_q;
        known = known && unsigned(b.seqs[i]) < unsigned(kv.max_seqs);
    }
    for (int g = tid; g < ng; g += kPlan) groups = groups && 0 <= b.cu_group[g] && b.cu_group[g] <= b.cu_group[g + 1] && b.cu_group[g + 1] <= b.n;
    if (!order || !groups || !known) atomicMin(kv.status, SIM_E_INVAL);
    order = __syncthreads_and(order);
    groups = __syncthreads_and(groups);
    const auto group_tokens = [&](int g) { return b.cu_q[b.cu_group[g + 1]] - b.cu_q[b.cu_group[g]]; };
    if (ng > 0) {
        for (int g = tid; g < ng; g += kPlan) {
            p.used[g] = INT_MAX;
            p.alone[g] = 0;
        }
        __syncthreads();
        for (int i0 = 0; i0 < b.n; i0 += kPlan) {  // the least number of pages of each group, the sum of its tile rows
            const int i = i0 + tid, g = i < b.n ? group_of(b, i) : -1, v = g < 0 ? INT_MAX : p.same[i];
            const int t = g < 0 ? 0 : tile_rows(entry_at(kv, b, i).t * G);
            int same_group;
            __match_all_sync(FULL, g, &same_group);
            if (same_group) {
                const int least = __reduce_min_sync(FULL, v), all = __reduce_add_sync(FULL, t);
                if (g >= 0 && (tid & 31) == 0) {
                    atomicMin(&p.used[g], least);
                    atomicAdd(&p.alone[g], all);
                }
            } else if (g >= 0) {
                atomicMin(&p.used[g], v);
                atomicAdd(&p.alone[g], t);
            }
        }
        __syncthreads();
        for (int g = tid; g < ng; g += kPlan) {
            // Sharing saves tiles, and costs every row a second partial result.
            const int rows = order && groups ? group_tokens(g) * G : 0, found = rows > 0 && p.used[g] != INT_MAX ? p.used[g] : 0;
            const int64_t saved = int64_t(found * P / kAttTile) * (p.alone[g] - tile_rows(rows));
            p.used[g] = saved > kShareCost * int64_t(ceil_div(rows, kAttRows / 2)) ? found : 0;
        }
        __syncthreads();
    }
    int64_t sum = 0;  // heavy items, light ones above
    for (int s0 = 0; s0 < n_src; s0 += kPlan) {
        const int s = s0 + tid;
        int rows = 0;
        if (s < ng) {
            if (p.used[s] > 0) rows = group_tokens(s) * G;
        } else if (s < n_src) {
            rows = order ? entry_at(kv, b, s - ng).t * G : 0;
            p.group[s - ng] = group_of(b, s - ng);
        }
        int64_t total;
        const int64_t before = sum + plan_scan(int64_t(light_items(rows)) << 32 | heavy_items(rows), sums, total);
        sum += total;
        if (s < n_src) {
            p.first[0][s] = int(before & 0xffffffff);
            p.first[1][s] = int(before >> 32);
        }
    }
    const int n_heavy = int(sum & 0xffffffff), n_light = int(sum >> 32);
    if (tid == 0) {
        p.first[0][n_src] = p.hdr[0] = n_heavy;
        p.first[1][n_src] = p.hdr[1] = n_light;
        p.hdr[8] = order;
    }
    __syncthreads();
    int64_t rows = 0;
    for (int light = 0; light < 2; ++light) {
        const int n_items = light ? n_light : n_heavy;
        const int32_t *first = p.first[light];
        int64_t units = 0, list_rows = 0;
        for (int k0 = 0; k0 < n_items; k0 += kPlan) {
            const int k = k0 + tid;
            KvItem it = {};
            if (k < n_items) {
                int lo = 0, hi = n_src;  // the last source that begins at or before item k
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (first[mid] <= k) lo = mid;
                    else hi = mid;
                }
                // a source's light item comes after its heavy ones
                const int in = light ? p.first[0][lo + 1] - p.first[0][lo] : k - first[lo];
                it.row0 = in * kAttRows;
                if (lo < ng) {
                    const int a = b.cu_group[lo];
                    it.q0 = b.cu_q[a];
                    it.rows = group_tokens(lo) * G - it.row0;
                    it.seq = b.seqs[a];
                    it.kv1 = p.used[lo] * P;
                    it.pos0 = 1 << 30;
                    it.partial = 1;
                    it.entry = -1;
                } else {
                    const Entry e = entry_at(kv, b, lo - ng);
                    const int g = p.group[lo - ng], shared = g < 0 ? 0 : p.used[g];
                    it.q0 = e.a;
                    it.rows = e.t * G - it.row0;
                    it.seq = e.seq;
                    it.kv0 = shared * P;
                    it.pos0 = e.len - e.t;
                    it.kv1 = min(e.len, it.pos0 + (it.row0 + min(it.rows, kAttRows) - 1) / G + 1);
                    it.partial = shared > 0;
                    it.entry = lo - ng;
                }
                it.rows = min(it.rows, light ? kAttRows / 2 : kAttRows);
                it.tiles = ceil_div(max(it.kv1 - it.kv0, 0), kAttTile);
            }
            int64_t total;
            it.unit = units + plan_scan(int64_t(it.tiles) * kv.n_kv_heads, sums, total);
            units += total;
            it.row_off = list_rows + plan_scan(int64_t(it.rows) * kv.n_kv_heads, sums, total);
            list_rows += total;
            if (k < n_items) p.items[light][k] = it;
        }
        if (tid == 0) *reinterpret_cast<int64_t *>(p.hdr + 2 + 2 * light) = units;
        rows += list_rows;
        if (tid == 0 && !light) *reinterpret_cast<int64_t *>(p.hdr + 6) = rows;
        __syncthreads();
        for (int c = tid; c < kv_blocks(sms, light); c += kPlan) {
            const int64_t u = line_at(units, c, kv_blocks(sms, light));
            int lo = 0, hi = n_items;  // the last item that begins at or before the block's stretch
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.items[light][mid].unit <= u) lo = mid;
                else hi = mid;
            }
            p.start[light][c] = lo;
        }
    }
}

// ---- the line of work ---------------------------------------------------------------------------------------

// First row of the partial results of block c's piece of a list whose rows follow `base` others.
__device__ __forceinline__ int64_t piece_row(const KvItem &it, int h, int c, int64_t base, int light) {
    return base + it.row_off + int64_t(h) * it.rows + int64_t(light ? kAttRows / 2 : kAttRows) * c;
}
__device__ __forceinline__ int64_t list_base(const KvPlan &p, int light, int sms) {
    return light ? *reinterpret_cast<const int64_t *>(p.hdr + 6) + int64_t(kAttRows) * kv_blocks(sms, 0) : 0;
}

// A stretch of one item and kv head, as the warps of a block pass it on.
struct alignas(16) Segment {
    int32_t n;               // tiles, 0: the end
    int32_t h;
    int32_t q0, row0, rows, pos0;
    int32_t k0, kv1;         // first key, end of the keys
    int32_t direct;          // results go to the output, not to the workspace
    int32_t pad;
    int64_t row;             // row of the partial results
};

// Walks the stretch of a list's line that is block c's.
struct Line {
    const KvItem *items;
    KvItem it;
    int64_t u, u1, base;
    int n_items, heads, k, h, c, light;
    __device__ Line(const KvPlan &p, int heads_, int light_, int c_, int sms) : items(p.items[light_]), heads(heads_), c(c_), light(light_) {
        n_items = p.hdr[light];
        const int64_t units = *reinterpret_cast<const int64_t *>(p.hdr + 2 + 2 * light);
        u = line_at(units, c, kv_blocks(sms, light));
        u1 = line_at(units, c + 1, kv_blocks(sms, light));
        base = list_base(p, light, sms);
        k = p.start[light][c];
        h = -1;
    }
    // The next item and head with work for this block; s.n = 0 at the end.
    __device__ void next(Segment &s) {
        s.n = 0;
        while (u < u1 && k < n_items) {
            if (h < 0) it = items[k];
            if (it.tiles == 0 || h + 1 == heads) {
                ++k;
                h = -1;
                continue;
            }
            h = h < 0 ? int((u - it.unit) / it.tiles) : h + 1;
            const int64_t a = it.unit + int64_t(h) * it.tiles;
            const int t0 = int(u - a), t1 = int(min(u1 - a, int64_t(it.tiles)));
            s.n = t1 - t0;
            s.h = h;
            s.q0 = it.q0;
            s.row0 = it.row0;
            s.rows = it.rows;
            s.pos0 = it.pos0;
            s.k0 = it.kv0 + t0 * kAttTile;
            s.kv1 = it.kv1;
            s.direct = s.n == it.tiles && !it.partial;
            s.row = piece_row(it, h, c, base, light);
            u = a + t1;
            return;
        }
    }
};

// ---- PTX ----------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
// Waits for the phase of that parity to end; gives up after about a second, or when another warp has.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    if (bar_try(bar, parity)) return true;
    const long long start = clock64();
    while (!bar_try(bar, parity)) {
        if (*gave_up) return false;
        if (clock64() - start > 2000000000LL) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(p));
    return p;
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z, int w) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void smem_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D (TMEM) = A (shared memory) B (shared memory), 16 of the inner dimension.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
        : "memory");
}
// A from TMEM.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
        : "memory");
}

#define REG4(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
#define VAL4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
__device__ __forceinline__ void tm_ld32(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : REG4(r, 0), REG4(r, 4), REG4(r, 8), REG4(r, 12), REG4(r, 16), REG4(r, 20), REG4(r, 24), REG4(r, 28)
        : "r"(addr));
}
__device__ __forceinline__ void tm_ld16(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : REG4(r, 0), REG4(r, 4), REG4(r, 8), REG4(r, 12)
        : "r"(addr));
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        VAL4(r, 0), VAL4(r, 4), VAL4(r, 8), VAL4(r, 12), VAL4(r, 16), VAL4(r, 20), VAL4(r, 24), VAL4(r, 28)
        : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
            addr),
        VAL4(r, 0), VAL4(r, 4), VAL4(r, 8), VAL4(r, 12)
        : "memory");
}
#undef REG4
#undef VAL4

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z, w;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 w, x, y, z;\n\t"
        "mov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, w;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 w, x, y;\n\t"
        "mov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
template <bool BF>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    if (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Shared-memory operand: 128-byte rows, 8 rows of 1024 bytes swizzled as one; `sbo` bytes between groups of 8
// rows, `lbo` between 64-column blocks where the long dimension is the contiguous one.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return uint64_t((addr >> 4) & 0x3fff) | uint64_t(lbo >> 4) << 16 | uint64_t(sbo >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

// ---- k_attend -----------------------------------------------------------------------------------------------

// HEAVY: 256 rows in two softmax groups that share every tile, one block per SM; otherwise 128 rows, one group,
// two blocks per SM.
template <int DP, bool HEAVY>
struct Shape {
    static constexpr int kGroups = HEAVY ? 2 : 1;
    static constexpr int kThreads = kGroups * 128 + 128;
    static constexpr int kTile = DP * 256;                                    // bytes of 128 query rows, or of a tile of keys or values
    static constexpr int kHalf = 16384;                                       // 128 rows of 64 columns
    static constexpr int kSlots = (HEAVY ? 131072 : 65536) / kTile;           // tiles of keys or values in flight
    static constexpr int kTmem = HEAVY ? 512 : 256;
    static constexpr int kOffO = kGroups * 128;                               // TMEM column of the first group's O
    static constexpr int kSoftRegs = HEAVY ? 208 : 184, kOtherRegs = HEAVY ? 88 : 72;
    // the launch gives 168 (128) registers a thread: no more are handed out
    static_assert(kGroups * kSoftRegs + kOtherRegs <= (kGroups + 1) * (HEAVY ? 168 : 128), "registers");
    static constexpr int kOffRing = kGroups * kTile;
    static constexpr int kOffStage = kOffRing + kSlots * kTile;
    static constexpr int kOffStat = kOffStage + kGroups * kStage * 4;
    static constexpr int kOffSeg = kOffStat + kGroups * 128 * 8;
    static constexpr int kOffBar = kOffSeg + kSegs * int(sizeof(Segment));
    static constexpr int kBars = 2 * kSlots + 2 * kSegs + 2 + 3 * kGroups + 2;
    static constexpr int kBytes = kOffBar + kBars * 8 + 16;
    static constexpr int kAlloc = kBytes + 1024;                              // the base is rounded up to 1024
    static_assert(kAlloc <= (HEAVY ? 232448 : 115712), "shared memory");
};

template <int DP, bool BF, bool HEAVY>
__global__ void __launch_bounds__(Shape<DP, HEAVY>::kThreads, HEAVY ? 1 : 2)
    k_attend(const sim_kv kv, const sim_kv_batch b, const KvAttend a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using Sh = Shape<DP, HEAVY>;
    constexpr int NS = Sh::kSlots, NG = Sh::kGroups;
    extern __shared__ unsigned char raw[];
    unsigned char *const base = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
    const uint32_t sbase = smem_addr(base), bars = sbase + Sh::kOffBar;
    volatile int *const gave_up = reinterpret_cast<int *>(base + Sh::kOffBar + Sh::kBars * 8);
    uint32_t *const tmem_at = reinterpret_cast<uint32_t *>(base + Sh::kOffBar + Sh::kBars * 8 + 4);
    Segment *const segs = reinterpret_cast<Segment *>(base + Sh::kOffSeg);
    const auto full = [&](uint32_t x) { return bars + 8 * (x % NS); };
    const auto empty = [&](uint32_t x) { return bars + 8 * (NS + x % NS); };
    const auto seg_full = [&](uint32_t x) { return bars + 8 * (2 * NS + x % kSegs); };
    const auto seg_empty = [&](uint32_t x) { return bars + 8 * (2 * NS + kSegs + x % kSegs); };
    constexpr int kRest = 2 * NS + 2 * kSegs;
    const uint32_t q_full = bars + 8 * kRest, q_empty = bars + 8 * (kRest + 1);
    const auto s_full = [&](int g) { return bars + 8 * (kRest + 2 + g); };
    const auto p_ready = [&](int g) { return bars + 8 * (kRest + 2 + NG + g); };
    const auto o_full = [&](int g) { return bars + 8 * (kRest + 2 + 2 * NG + g); };
    const uint32_t drained = bars + 8 * (kRest + 2 + 3 * NG), joined = drained + 8;
    const int tid = threadIdx.x, warp = __shfl_sync(FULL, tid >> 5, 0), lane = tid & 31, role = warp - 4 * NG;

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int s = 0; s < kSegs; ++s) {
            bar_init(seg_full(s), 1);
            bar_init(seg_empty(s), 4 * NG + 3);
        }
        bar_init(q_full, 2);
        bar_init(q_empty, 1);
        for (int g = 0; g < NG; ++g) {
            bar_init(s_full(g), 1);
            bar_init(p_ready(g), 4);
            bar_init(o_full(g), 1);
        }
        bar_init(drained, 1);
        bar_init(joined, 4);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (role == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_at)), "n"(Sh::kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(FULL, *tmem_at, 0);
    kv_wait_previous();

    const int G = b.q_heads / kv.n_kv_heads, D = kv.head_dim;
    // Segment number x, for the warps that are told of it; empty if the wait gave up.
    const auto take = [&](uint32_t x, Segment &s) {
        const bool ok = __all_sync(FULL, bar_wait(seg_full(x), (x / kSegs) & 1, gave_up));
        if (ok) s = segs[x % kSegs];
        else s.n = 0;
        __syncwarp();
        if (lane == 0) bar_arrive(seg_empty(x));
        return ok;
    };

    if (role >= 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kOtherRegs));
        if (role == 0) {
            // ---- the line of work, and loads: lane l brings page l of each tile
            const KvPlan plan = kv_plan(kv, b);
            Line line(plan, kv.n_kv_heads, HEAVY ? 0 : 1, blockIdx.x, a.sms);
            const int P = kv.page_size, per = kAttTile / P;
            uint32_t at = 0;  // tiles loaded
            bool ok = true;
            for (uint32_t x = 0; ok; ++x) {
                Segment sg;
                line.next(sg);
                ok = __all_sync(FULL, bar_wait(seg_empty(x), (x / kSegs + 1) & 1, gave_up));
                if (!ok) break;
                if (lane == 0) {
                    segs[x % kSegs] = sg;
                    bar_arrive(seg_full(x));
                }
                if (sg.n == 0) break;
                const int32_t *row = kv.table + int64_t(line.it.seq) * kv.max_pages;
                const int first = sg.k0 / P + lane;
                const auto page_of = [&](int j) {  // of this lane in tile j; past the keys: none, zeros
                    const int idx = first + j * per;
                    return lane < per && j < sg.n && idx * P < sg.kv1 ? row[idx] : -1;
                };
                int page = page_of(0);
                for (int j = 0; j < sg.n && ok; ++j) {
                    const int next_page = page_of(j + 1);
                    const int w = unsigned(page) < unsigned(kv.n_pages) ? page : kv.n_pages;
#pragma unroll
                    for (int v = 0; v < 2; ++v, ++at) {  // keys, values
                        ok = __all_sync(FULL, bar_wait(empty(at), (at / NS + 1) & 1, gave_up));
                        if (!ok) break;
                        if (lane == 0) bar_expect(full(at), Sh::kTile);
                        __syncwarp();
                        if (lane < per) {
                            const uint32_t dst = sbase + Sh::kOffRing + (at % NS) * Sh::kTile + lane * P * 128;
#pragma unroll
                            for (int half = 0; half < DP / 64; ++half)
                                tma_load(dst + half * Sh::kHalf, v ? &map_v : &map_k, full(at), half * 64, 0, sg.h, w);
                        }
                    }
                    page = next_page;
                }
            }
            if (!ok) {  // let what is on its way arrive
                for (uint32_t k = at > NS ? at - NS : 0; k < at; ++k)
                    for (int n = 0; n < 1000000 && !bar_try(full(k), (k / NS) & 1); ++n) {
                    }
                if (lane == 0) atomicMin(kv.status, SIM_E_STATE);
            }
        } else if (role == 1) {
            // ---- tensor products: the whole warp keeps the same (uniform) state, one lane issues
            const uint32_t type = BF ? 1u << 7 | 1u << 10 : 0u;
            const uint32_t idesc_s = 1u << 4 | type | (128 / 8) << 17 | (128 / 16) << 24;
            const uint32_t idesc_o = 1u << 4 | type | 1u << 16 | (DP / 8) << 17 | (128 / 16) << 24;
            const uint64_t op_q = operand(sbase, 16, 1024), op_k = operand(sbase + Sh::kOffRing, 16, 1024), op_v = operand(sbase + Sh::kOffRing, Sh::kHalf, 1024);
            uint32_t at = 0, np = 0;
            bool ok = true;
            const auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(FULL, bar_wait(bar, parity, gave_up)) != 0; };
            const auto wait_full = [&](uint32_t y) { return wait(full(y), (y / NS) & 1); };
            Segment sg;
            for (uint32_t x = 0; (ok = take(x, sg)); ++x) {
                const int n = __shfl_sync(FULL, sg.n, 0);
                if (n == 0) break;
                const auto keys = [&](int j, int g) {  // S of group g and tile j
                    if (elect_one()) {
                        const uint32_t slot = (at + 2 * j) % NS;
#pragma unroll
                        for (int kk = 0; kk < DP / 16; ++kk) {
                            const uint32_t off = (kk / 4) * Sh::kHalf + (kk % 4) * 32;
                            mma_ss(tmem + g * 128, op_q + ((g * Sh::kTile + off) >> 4), op_k + ((slot * Sh::kTile + off) >> 4), idesc_s, kk > 0);
                        }
                        tc_commit(s_full(g));
                        if (g == NG - 1) {
                            tc_commit(empty(at + 2 * j));
                            if (j == n - 1) tc_commit(q_empty);
                        }
                    }
                    __syncwarp();
                };
                ok = wait(q_full, x & 1) && wait_full(at);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int g = 0; g < NG; ++g) keys(0, g);
                for (int j = 0; j < n && ok; ++j, ++np) {
                    ok = wait_full(at + 2 * j + 1);
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        ok = ok && wait(p_ready(g), np & 1);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t slot = (at + 2 * j + 1) % NS;
#pragma unroll
                            for (int kk = 0; kk < kAttTile / 16; ++kk)
                                mma_ts(tmem + Sh::kOffO + g * 128, tmem + g * 128 + kk * 8, op_v + ((slot * Sh::kTile + kk * 2048) >> 4), idesc_o, j > 0 || kk > 0);
                            if (g == NG - 1) tc_commit(empty(at + 2 * j + 1));
                            if (j + 1 == n) tc_commit(o_full(g));
                        }
                        __syncwarp();
                        if (j + 1 < n) {
                            if (g == 0) ok = wait_full(at + 2 * j + 2);
                            if (!ok) break;
                            keys(j + 1, g);
                        }
                    }
                }
                if (!ok) break;
                at += 2 * n;
            }
            if (!ok) {
                if (elect_one()) {
                    tc_commit(drained);
                    atomicMin(kv.status, SIM_E_STATE);
                }
                __syncwarp();
                for (int n = 0; n < 1000000 && !bar_try(drained, 0); ++n) {
                }
            }
            __syncwarp();
        } else {
            // ---- query rows: two warps, 16 bytes a lane, the lanes of a row side by side.  Rows past the item's are
            // left as they are: what they hold meets no other row and is masked.
            constexpr int kVec = DP / 8, kStep = 64 / kVec;
            const int j = (tid & 63) % kVec;
            const bool has = j * 8 < D;
            Segment sg;
            for (uint32_t x = 0; take(x, sg) && sg.n > 0; ++x) {
                // 64 (32) rows or fewer lie in the tile twice (four times)
                const int span = HEAVY ? 256 : sg.rows > 64 ? 128 : sg.rows > 32 ? 64 : 32;
                const uint16_t *const from0 = static_cast<const uint16_t *>(a.q) + int64_t(sg.q0) * a.qt + int64_t(sg.h * G) * a.qh + (has ? j * 8 : 0);
                if (!__all_sync(FULL, bar_wait(q_empty, (x + 1) & 1, gave_up))) break;
#pragma unroll 4
                for (int r = (tid & 63) / kVec; r < sg.rows; r += kStep) {
                    const int y = sg.row0 + r, t = a.group.div(y);
                    const uint16_t *from = from0 + int64_t(t) * a.qt + int64_t(y - t * G) * a.qh;
                    const uint32_t to = sbase + (r >> 7) * Sh::kTile + (j / 8) * Sh::kHalf + (r & 127) * 128 + (((j % 8) ^ (r & 7)) << 4);
                    if (a.q_vec) {
                        const int bytes = has ? 16 : 0;  // columns past the head's are zeros
                        for (int c = 0; c < 128; c += span)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + c * 128), "l"(from), "r"(bytes) : "memory");
                    } else {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (has)
                            v = make_uint4(from[0] | uint32_t(from[1]) << 16, from[2] | uint32_t(from[3]) << 16, from[4] | uint32_t(from[5]) << 16,
                                           from[6] | uint32_t(from[7]) << 16);
                        for (int c = 0; c < 128; c += span)
                            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to + c * 128), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                smem_to_async();
                __syncwarp();
                if (lane == 0) bar_arrive(q_full);
            }
        }
    } else {
        // ---- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kSoftRegs));
        const int g = warp >> 2, w = warp & 3, lr = tid & 127;
        const uint32_t t_lane = tmem + (uint32_t(w * 32) << 16), t_s = t_lane + g * 128, t_o = t_lane + Sh::kOffO + g * 128;
        float *const stage = reinterpret_cast<float *>(base + Sh::kOffStage) + g * kStage;
        float2 *const stat = reinterpret_cast<float2 *>(base + Sh::kOffStat) + g * 128;
        const float c = a.scale_log2, grow = kGrow / c;
        uint32_t ns = 0, nj = 0, at = 0;
        bool ok = true;
        const auto join = [&] {  // the group's warps, by a barrier whose wait ends even if some have given up
            __syncwarp();
            if (lane == 0) bar_arrive(joined);
            ok = __all_sync(FULL, bar_wait(joined, nj++ & 1, gave_up)) && ok;
        };
        Segment sg;
        for (uint32_t x = 0; ok && take(x, sg) && sg.n > 0; ++x) {
            const int rows = sg.rows;
            const int r = HEAVY ? g * 128 + lr : rows > 64 ? lr : rows > 32 ? lr & 63 : lr & 31;  // the row in this thread's lane
            const int last = r < rows ? min(sg.kv1 - 1, sg.pos0 + int(a.group.div(sg.row0 + r))) : -1;  // key position that it sees last
            float m = -INFINITY, l = 0.f;

            const auto tiles = [&](auto copies) {
                constexpr int R = decltype(copies)::value, NC = 128 / R;  // columns per thread
                const int c0 = R == 4 ? w * 32 : R == 2 ? (w >> 1) * 64 : 0;
                for (int j = 0; j < sg.n; ++j) {
                    const int k0 = sg.k0 + j * kAttTile;  // first key of the tile
                    ok = __all_sync(FULL, bar_wait(s_full(g), ns & 1, gave_up));
                    if (!ok) return;
                    ++ns;
                    tc_fence_after();
                    uint32_t s[NC];
#pragma unroll
                    for (int q = 0; q < NC / 32; ++q) tm_ld32(t_s + c0 + 32 * q, s + 32 * q);
                    tc_wait_ld();
                    const int lim = last - k0 - c0;  // column of this thread that the row sees last
                    if (__any_sync(FULL, lim < NC - 1)) {
#pragma unroll
                        for (int y = 0; y < NC; ++y)
                            if (y > lim) s[y] = 0xff800000u;
                    }
                    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int y = 0; y < NC; y += 2) top[y / 2 & 3] = max3(top[y / 2 & 3], __uint_as_float(s[y]), __uint_as_float(s[y + 1]));
                    const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                    if (j == 0) {
                        m = mx;
                    } else if (__any_sync(FULL, mx > m + grow)) {
                        const float up = fmaxf(m, mx), f = up == m ? 1.f : ex2((m - up) * c);
                        m = up;
                        l *= f;
#pragma unroll
                        for (int q = 0; q < DP / 32; ++q) {
                            uint32_t o[32];
                            tm_ld32(t_o + 32 * q, o);
                            tc_wait_ld();
#pragma unroll
                            for (int y = 0; y < 32; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * f);
                            tm_st32(t_o + 32 * q, o);
                        }
                    }
                    const float off = m == -INFINITY ? 0.f : m * c;
                    float2 sum[4] = {};
                    uint32_t pk[NC / 2];
#pragma unroll
                    for (int y = 0; y < NC; y += 2) {
                        float2 e = fma2(make_float2(__uint_as_float(s[y]), __uint_as_float(s[y + 1])), make_float2(c, c), make_float2(-off, -off));
                        e = make_float2(ex2(e.x), ex2(e.y));
                        sum[y / 2 & 3] = add2(sum[y / 2 & 3], e);
                        pk[y / 2] = pack<BF>(e.x, e.y);
                    }
                    sum[0] = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
                    l += sum[0].x + sum[0].y;
                    if constexpr (R == 1) {
                        tm_st32(t_s, pk);
                        tm_st32(t_s + 32, pk + 32);
                    } else if constexpr (R == 2) {
                        uint32_t z[32];
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
#pragma unroll
                            for (int y = 0; y < 32; ++y) z[y] = q == (w >> 1) ? pk[y] : 0;
                            tm_st32(t_s + 32 * q, z);
                        }
                    } else {
                        uint32_t z[16];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
#pragma unroll
                            for (int y = 0; y < 16; ++y) z[y] = q == w ? pk[y] : 0;
                            tm_st16(t_s + 16 * q, z);
                        }
                    }
                    tc_wait_st();
                    // values past the end of the keys, whatever they are, must not meet their zero probabilities
                    const int valid = sg.kv1 - k0;
                    if (valid < kAttTile && g == 0) {
                        const uint32_t y = at + 2 * j + 1;
                        ok = __all_sync(FULL, bar_wait(full(y), (y / NS) & 1, gave_up));
                        if (lr >= valid) {
                            unsigned char *v = base + Sh::kOffRing + (y % NS) * Sh::kTile + lr * 128;
#pragma unroll
                            for (int z = 0; z < DP / 8; ++z) *reinterpret_cast<uint4 *>(v + (z / 8) * Sh::kHalf + (z % 8) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        smem_to_async();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_ready(g));
                }
            };
            if (HEAVY || rows > 64) tiles(std::integral_constant<int, 1>());
            else if (rows > 32) tiles(std::integral_constant<int, 2>());
            else tiles(std::integral_constant<int, 4>());
            if (!ok) break;
            at += 2 * sg.n;

            const auto out_row = [&](int y) {  // of row y of the item
                const int t = a.group.div(sg.row0 + y);
                return static_cast<uint16_t *>(a.out) + int64_t(sg.q0 + t) * a.ot + int64_t(sg.h * G + (sg.row0 + y - t * G)) * a.oh;
            };
            const auto put_lse = [&](int y, float top, float total) {
                const float e = total == 0.f ? -INFINITY : top * c + log2f(total);
                if (!sg.direct) {
                    a.part_lse[sg.row + y] = e;
                } else if (a.lse) {
                    const int t = a.group.div(sg.row0 + y);
                    a.lse[int64_t(sg.q0 + t) * b.q_heads + sg.h * G + (sg.row0 + y - t * G)] = e * 0.69314718055994531f;
                }
            };
            float f;  // what this thread's part of O is multiplied by
            const int span = HEAVY || rows > 64 ? 128 : rows > 32 ? 64 : 32;
            if (span == 128) {
                f = l == 0.f ? 0.f : 1.f / l;
                if (r < rows) put_lse(r, m, l);
            } else {
                stat[lr] = make_float2(m, l);
                join();
                const int row = lr & (span - 1);
                float top = -INFINITY, total = 0.f;
                for (int p = row; p < 128; p += span)
                    if (stat[p].y != 0.f) top = fmaxf(top, stat[p].x);
                for (int p = row; p < 128; p += span)
                    if (stat[p].y != 0.f) total += stat[p].y * ex2((stat[p].x - top) * c);
                f = l == 0.f ? 0.f : ex2((m - top) * c) / total;
                if (lr < min(span, rows)) put_lse(lr, top, total);
            }
            ok = __all_sync(FULL, bar_wait(o_full(g), x & 1, gave_up)) && ok;
            if (!ok) break;
            tc_fence_after();
            if (span == 128) {  // each warp by itself: 16 columns of its 32 rows at a time, so that stores fill sectors
                float *const mine = stage + w * 32 * 17;
                const int row0 = r - lane;
                for (int d0 = 0; d0 < DP && d0 < D; d0 += 16) {
                    uint32_t o[16];
                    tm_ld16(t_o + d0, o);
                    tc_wait_ld();
#pragma unroll
                    for (int y = 0; y < 16; ++y) mine[lane * 17 + y] = l == 0.f ? 0.f : __uint_as_float(o[y]) * f;
                    __syncwarp();
                    if (sg.direct) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int y = q * 16 + lane / 2, d = lane % 2 * 8;
                            const float *v = mine + y * 17 + d;
                            if (row0 + y < rows && d0 + d < D)
                                *reinterpret_cast<uint4 *>(out_row(row0 + y) + d0 + d) = make_uint4(pack<BF>(v[0], v[1]), pack<BF>(v[2], v[3]), pack<BF>(v[4], v[5]), pack<BF>(v[6], v[7]));
                        }
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int y = q * 8 + lane / 4, d = lane % 4 * 4;
                            const float *v = mine + y * 17 + d;
                            if (row0 + y < rows && d0 + d < D)
                                *reinterpret_cast<float4 *>(a.part + (sg.row + row0 + y) * D + d0 + d) = make_float4(v[0], v[1], v[2], v[3]);
                        }
                    }
                    __syncwarp();
                }
            } else {  // join the copies of each row, as many columns at a time as the stage holds of all of them
                const int parts = 128 / span;
                int cols = 16, shift = 3;
                while (cols < DP && parts * rows * (2 * cols + 1) <= kStage) {
                    cols *= 2;
                    ++shift;
                }
                const int row = lr & (span - 1), part = lr / span;
                for (int d0 = 0; d0 < D && ok; d0 += cols) {
                    for (int d = 0; d < cols; d += 16) {
                        uint32_t o[16];
                        tm_ld16(t_o + d0 + d, o);
                        tc_wait_ld();
                        if (row < rows) {
#pragma unroll
                            for (int y = 0; y < 16; ++y) stage[(part * rows + row) * (cols + 1) + d + y] = l == 0.f ? 0.f : __uint_as_float(o[y]) * f;
                        }
                    }
                    join();
                    for (int e = lr; e < rows << shift; e += 128) {
                        const int y = e >> shift, d = 2 * (e & ((1 << shift) - 1));
                        if (d0 + d >= D) continue;
                        float v0 = 0.f, v1 = 0.f;
                        for (int p = 0; p < parts; ++p) {
                            const float *v = stage + (p * rows + y) * (cols + 1) + d;
                            v0 += v[0];
                            v1 += v[1];
                        }
                        if (sg.direct) *reinterpret_cast<uint32_t *>(out_row(y) + d0 + d) = pack<BF>(v0, v1);
                        else *reinterpret_cast<float2 *>(a.part + (sg.row + y) * D + d0 + d) = make_float2(v0, v1);
                    }
                    join();
                }
            }
            tc_fence_before();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (role == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Sh::kTmem));
    }
}

// ---- k_combine ----------------------------------------------------------------------------------------------

// The pieces of one item and head: those of blocks c0 .. c1 that have any of its tiles.
struct Pieces {
    int64_t row, units;
    int c0, n, blocks, rows;
    __device__ Pieces() : row(0), units(0), c0(0), n(0), blocks(1), rows(0) {}
    __device__ Pieces(const KvPlan &p, const KvItem &it, int h, int light, int sms) : units(0), c0(0), n(0), blocks(kv_blocks(sms, light)) {
        rows = light ? kAttRows / 2 : kAttRows;
        if (it.tiles > 0) {
            units = *reinterpret_cast<const int64_t *>(p.hdr + (light ? 4 : 2));
            const int64_t from = it.unit + int64_t(h) * it.tiles;
            c0 = block_at(units, from, blocks);
            n = block_at(units, from + it.tiles - 1, blocks) - c0 + 1;
        }
        row = piece_row(it, h, c0, list_base(p, light, sms), light);
    }
    // Row `in` of the item in piece i, -1 if the block has none of its tiles (where there are fewer tiles than blocks).
    __device__ int64_t at(int i, int in) const {
        const bool some = units >= blocks || line_at(units, c0 + i, blocks) < line_at(units, c0 + i + 1, blocks);
        return i >= 0 && i < n && some ? row + int64_t(rows) * i + in : -1;
    }
};

// Rows whose keys were divided among items or blocks, or that see none: a block for 32 rows of an entry's item
// and one head, eight lanes for each row.  The lanes first read the sums of eight pieces, then, without waiting
// in between, those pieces' columns.
template <bool BF>
__global__ void __launch_bounds__(256) k_combine(const sim_kv kv, const sim_kv_batch b, const KvAttend a) {
    kv_wait_previous();
    const KvPlan plan = kv_plan(kv, b);
    const int H = kv.n_kv_heads, G = b.q_heads / H, D = kv.head_dim, sub = (threadIdx.x & 31) >> 3, sl = threadIdx.x & 7, warp = threadIdx.x >> 5;
    const auto put = [&](int t, int qh, const float4 *v, float f, float lse) {
        uint16_t *o = static_cast<uint16_t *>(a.out) + int64_t(t) * a.ot + int64_t(qh) * a.oh;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = 4 * (sl + 8 * q);
            if (d < D) *reinterpret_cast<uint2 *>(o + d) = make_uint2(pack<BF>(v[q].x * f, v[q].y * f), pack<BF>(v[q].z * f, v[q].w * f));
        }
        if (sl == 0 && a.lse) a.lse[int64_t(t) * b.q_heads + qh] = lse;
    };
    const int heavy0 = plan.first[0][b.n_groups], light0 = plan.first[1][b.n_groups];
    const int64_t heavy = int64_t(plan.hdr[0] - heavy0) * H * 8, all = heavy + int64_t(plan.hdr[1] - light0) * H * 4;
    for (int64_t x = blockIdx.x; x < all; x += gridDim.x) {
        const bool light = x >= heavy;
        const uint32_t y = uint32_t(light ? x - heavy : x), ih = light ? y >> 2 : y >> 3;
        const int r0 = 32 * int(light ? y & 3 : y & 7), k = int(ih / H), h = int(ih % H);
        const KvItem *const at_item = light ? plan.items[1] + light0 + k : plan.items[0] + heavy0 + k;
        if (r0 >= at_item->rows) continue;
        const KvItem it = *at_item;
        const Pieces own(plan, it, h, light, a.sms);
        if (own.n == 1 && !it.partial) continue;  // k_attend wrote these rows
        const int r = r0 + warp * 4 + sub;
        const bool row = r < it.rows;
        const int z = it.row0 + min(r, it.rows - 1), t = it.q0 + int(a.group.div(z)), qh = h * G + z - (t - it.q0) * G;
        Pieces prefix;
        int in = 0;
        if (it.partial) {
            const int g = plan.group[it.entry], nth_row = (t - b.cu_q[b.cu_group[g]]) * G + qh - h * G, nth = nth_row / kAttRows, h0 = plan.first[0][g];
            const bool l = nth >= plan.first[0][g + 1] - h0;
            prefix = Pieces(plan, l ? plan.items[1][plan.first[1][g]] : plan.items[0][h0 + nth], h, l, a.sms);
            in = nth_row % kAttRows;
        }
        const int n = prefix.n + own.n, most = int(__reduce_max_sync(FULL, unsigned(n)));
        float top = -INFINITY, total = 0.f;
        float4 acc[4] = {};
        for (int p0 = 0; p0 < most; p0 += 8) {
            const int p = p0 + sl;
            const int64_t at = p < prefix.n ? prefix.at(p, in) : own.at(p - prefix.n, min(r, it.rows - 1));
            const float s = at >= 0 ? a.part_lse[at] : -INFINITY;
            float up = s;
#pragma unroll
            for (int d = 4; d >= 1; d >>= 1) up = fmaxf(up, __shfl_xor_sync(FULL, up, d));
            up = fmaxf(up, top);
            const float w = s == -INFINITY ? 0.f : ex2(s - up), f = top == -INFINITY ? 0.f : ex2(top - up);
            top = up;
            total *= f;
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[q] = make_float4(acc[q].x * f, acc[q].y * f, acc[q].z * f, acc[q].w * f);
#pragma unroll
            for (int i0 = 0; i0 < 8; i0 += 4) {
                if (p0 + i0 >= most) break;
                float4 v[4][4];  // a piece that is not there: row 0, with weight 0
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 *from = reinterpret_cast<const float4 *>(a.part + max(__shfl_sync(FULL, at, i0 + i, 8), int64_t(0)) * D);
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[i][q] = __ldcs(from + (4 * (sl + 8 * q) < D ? sl + 8 * q : 0));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float wi = __shfl_sync(FULL, w, i0 + i, 8);
                    total += wi;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float4 x = v[i][q];
                        acc[q] = wi == 0.f ? acc[q] : make_float4(fmaf(x.x, wi, acc[q].x), fmaf(x.y, wi, acc[q].y), fmaf(x.z, wi, acc[q].z), fmaf(x.w, wi, acc[q].w));
                    }
                }
            }
        }
        if (row) put(t, qh, acc, total == 0.f ? 0.f : 1.f / total, total == 0.f ? -INFINITY : (top + log2f(total)) * 0.69314718055994531f);
    }
    // query tokens of no entry
    const bool order = b.n > 0 && plan.hdr[8];
    const int first = order ? b.cu_q[0] : b.n_q, last = order ? b.cu_q[b.n] : b.n_q;
    const int64_t rest = int64_t(first + b.n_q - last) * b.q_heads;
    const float4 zero[4] = {};
    for (int64_t x = int64_t(blockIdx.x) * 32 + warp * 4 + sub; x < rest; x += int64_t(gridDim.x) * 32) {
        const int i = int(x / b.q_heads);
        put(i < first ? i : i - first + last, int(x % b.q_heads), zero, 0.f, -INFINITY);
    }
}

using EncodeFn = decltype(&cuTensorMapEncodeTiled);
EncodeFn encode_fn() {
    static EncodeFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

template <int DP, bool BF>
cudaError_t attend(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    // [page][head][token][dim] of one layer's keys, and of its values; boxes of one page and head, 64 columns
    const EncodeFn encode = encode_fn();
    if (!encode) return cudaErrorNotSupported;
    CUtensorMap maps[2];
    for (int v = 0; v < 2; ++v) {
        uint16_t *at = static_cast<uint16_t *>(kv.pool) + a.layer * kv_layer_elems(kv) + v * (kv_layer_elems(kv) / 2);
        const cuuint64_t dim[4] = {cuuint64_t(kv.head_dim), cuuint64_t(kv.page_size), cuuint64_t(kv.n_kv_heads), cuuint64_t(kv.n_pages)};
        const cuuint64_t stride[3] = {cuuint64_t(kv.head_dim) * 2, cuuint64_t(kv.head_dim) * 2 * kv.page_size, cuuint64_t(kv_page_bytes(kv))};
        const cuuint32_t box[4] = {64, cuuint32_t(kv.page_size), 1, 1}, step[4] = {1, 1, 1, 1};
        if (encode(&maps[v], BF ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, at, dim, stride, box, step,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    const auto heavy = k_attend<DP, BF, true>, light = k_attend<DP, BF, false>;
    static thread_local int ready = -1;  // the device whose kernels have their shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev != ready) {
        e = cudaFuncSetAttribute((const void *)heavy, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP, true>::kAlloc);
        if (e == cudaSuccess) e = cudaFuncSetAttribute((const void *)light, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP, false>::kAlloc);
        if (e == cudaSuccess) ready = dev;
    }
    if (e != cudaSuccess) return e;
    const int64_t rows = int64_t(b.n_q) * b.q_heads;
    if (rows / kv.n_kv_heads > kAttRows / 2)  // fewer rows make no heavy item
        e = launch_chained(heavy, kv_blocks(a.sms, 0), Shape<DP, true>::kThreads, Shape<DP, true>::kAlloc, st, kv, b, a, maps[0], maps[1]);
    if (e == cudaSuccess)
        e = launch_chained(light, kv_blocks(a.sms, 1), Shape<DP, false>::kThreads, Shape<DP, false>::kAlloc, st, kv, b, a, maps[0], maps[1]);
    if (e != cudaSuccess) return e;
    return launch_chained(k_combine<BF>, int(std::min<int64_t>(rows, int64_t(a.sms) * 8)), 256, 0, st, kv, b, a);
}

}  // namespace

cudaError_t launch_kv_plan(const sim_kv &kv, const sim_kv_batch &b, cudaStream_t st) {
    if (b.n_groups > 0) {
        cudaError_t e = launch_chained(k_plan_shared, std::max((b.n + 7) / 8, 1), 256, 0, st, kv, b);
        if (e != cudaSuccess) return e;
    }
    return launch_chained(k_plan_items, 1, kPlan, 0, st, kv, b, kv_sm_count());
}

cudaError_t launch_kv_attend(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    if (kv.dtype == SIM_KV_BF16) return kv.head_dim > 64 ? attend<128, true>(kv, b, a, st) : attend<64, true>(kv, b, a, st);
    return kv.head_dim > 64 ? attend<128, false>(kv, b, a, st) : attend<64, false>(kv, b, a, st);
}

}  // namespace simgb
