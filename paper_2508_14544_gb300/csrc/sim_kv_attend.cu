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
// The plan (k_plan_shared, k_plan_items, made once for all layers) lists the items.  Those of more than 32 rows
// are heavy, the others light: two kernels (sim_kv_heavy.cu, sim_kv_light.cu), because many rows want the tensor
// products fed and few rows want bytes in flight.  Measured either way, 8 kv heads (these and the figures below: plan and
// attention as a captured graph, caches flushed): 200 sequences of up to 2600 keys with 16 rows take 206 us light and 222 us
// heavy, 64 sequences of 2048 keys with 32 rows 124 and 126 us; a light item has no room for more.  The tiles of all items and heads of a list lie on one line, and every block takes an equal stretch of it, so that work
// is even whatever the lengths; an item is split where two stretches meet, and k_combine joins the pieces.  What taking up an
// item costs lies on the line too (kv_lead): left out, a step of 384 sequences takes 360 instead of 347 us and one of 256
// on a prefix 162 instead of 149 us.
#include <algorithm>

#include "sim_kv_attend.cuh"

namespace simgb {

namespace {

// ---- plan ---------------------------------------------------------------------------------------------------

// What sharing a prefix costs, in the time that a block needs for 128 keys: for the prefix's own item, for 32 rows that are
// then joined from two places, and for every block once (a longer chain of kernels).  Measured with and without sharing, 128
// sequences (8 kv heads, 8 query heads each, up to 64 keys of their own) in groups: 64 groups with a prefix of 512 keys 93
// against 71 us, of 2048 keys 140 against 170 us; 16 groups with 256 keys 72 against 52 us, with 1024 keys 75 against 81 us.
// The rule takes the faster side of these four.  With 2 kv heads of 4 query heads and D = 64 it shares a little early: 64 groups with
// 2048 keys 59 against 50 us (8192: 88 against 102), 16 groups with 1024 keys 48 against 42 us (4096: 59 against 63).
constexpr int kShareItem = 3, kShareRows = 7, kShareOnce = 2;

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

constexpr int kAhead = 16;  // 256 tables of 540 pages: the whole call takes 5 us less than with 2

// A warp for each entry: the pages that its table begins with like that of its group's first entry, all of whose
// keys each of its queries sees.  Bound by the latency of loads, so kAhead of either table are in flight: 5 us for 256 tables of
// 540 pages.
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
        for (int j0 = 0; j0 < most; j0 += 32 * kAhead) {  // that many loads of either table in flight
            int32_t u[kAhead], v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int j = j0 + 32 * k + lane;
                u[k] = j < most ? x[j] : 0;
                v[k] = j < most ? y[j] : 0;
            }
            int at = INT_MAX;
#pragma unroll
            for (int k = kAhead - 1; k >= 0; --k) {
                const unsigned m = __ballot_sync(FULL, u[k] != v[k]);
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

// Exclusive prefix sums of two values per thread over W warps, and the totals.
struct Two {
    int64_t a, b;
};
template <int W>
__device__ __forceinline__ Two plan_scan(Two v, Two *sums, Two &total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    Two x = v;
#pragma unroll 1
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t y = __shfl_up_sync(FULL, x.a, d), z = __shfl_up_sync(FULL, x.b, d);
        if (lane >= d) x = {x.a + y, x.b + z};
    }
    if (lane == 31) sums[w] = x;
    __syncthreads();
    Two before = {0, 0};
    total = {0, 0};
#pragma unroll 8
    for (int k = 0; k < W; ++k) {  // faster than a second scan by shuffles
        if (k == w) before = total;
        total = {total.a + sums[k].a, total.b + sums[k].b};
    }
    __syncthreads();
    return {before.a + x.a - v.a, before.b + x.b - v.b};
}

// Tile rows of 128 that r query rows take: two where they are more than 128 in their block of 256.
__device__ __forceinline__ int tile_rows(int r) {
    const int rem = r % kAttRows;
    return 2 * (r / kAttRows) + (rem > kAttRows / 2 ? 2 : rem > 0);
}
__device__ __forceinline__ int heavy_items(int r, bool only) { return only ? 0 : r / kAttRows + (r % kAttRows > kLightRows); }
__device__ __forceinline__ int light_items(int r, bool only) {
    return only ? ceil_div(r, kLightRows) : r % kAttRows > 0 && r % kAttRows <= kLightRows;
}

constexpr int kFewSources = 448, kFewItems = 1024;

// The last of n + 1 ascending numbers x[0] .. x[n] that is at most v, below n.
template <typename T>
__device__ __forceinline__ int last_at_most(const T *x, int n, T v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (x[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

// One block: which prefixes are shared, the sources and items, and where each begins on its list's line of work.
// Bound by its chain of dependent loads and barriers, not by bytes: 7 us for 40 entries, 12 us for 256 and their group.
// FEW: what the searches read is in shared memory, as far as that goes without asking for more than 48 KB; steps of 40, 64,
// 256 (on a prefix) and 440 sequences take 26, 33, 149 and 96 us in all, and 30, 36, 155 and 100 us without.
template <bool FEW>
__global__ void __launch_bounds__(FEW ? 512 : 1024) k_plan_items(const sim_kv kv, const sim_kv_batch b, int sms) {
    constexpr int kPlan = FEW ? 512 : 1024;
    __shared__ Two sums[32];
    __shared__ int32_t counts[3];  // cuts of heavy, of light items, entries to join
    __shared__ unsigned long long saved;
    __shared__ KvSource few_sources[FEW ? kFewSources : 1];
    __shared__ int32_t few_first[FEW ? 2 : 1][FEW ? kFewSources + 1 : 1], few_used[FEW ? kFewSources : 1], few_alone[FEW ? kFewSources : 1];
    __shared__ int64_t few_units[FEW ? kFewItems : 1];
    __shared__ int32_t few_tiles[FEW ? kFewItems : 1];  // -1: its results are not joined here
    kv_wait_previous();
    const KvPlan p = kv_plan(kv, b);
    KvSource *const source = FEW ? few_sources : p.source;
    int32_t *const used = FEW ? few_used : p.used, *const alone = FEW ? few_alone : p.alone;
    int32_t *const first0 = FEW ? few_first[0] : p.first[0], *const first1 = FEW ? few_first[FEW ? 1 : 0] : p.first[1];
    const int tid = threadIdx.x, ng = b.n_groups, n_src = ng + b.n, G = b.q_heads / kv.n_kv_heads, P = kv.page_size;
    const bool only = kv_light_only(kv, b);
    if (tid < 3) counts[tid] = 0;
    if (tid == 0) saved = 0;
    // Offsets that are not in order: no queries at all, or no groups.
    bool order = true, groups = true, known = true;
#pragma unroll 1
    for (int i = tid; i < b.n; i += kPlan) {
        order = order && 0 <= b.cu_q[i] && b.cu_q[i] <= b.cu_q[i + 1] && b.cu_q[i + 1] <= b.n_q;
        known = known && unsigned(b.seqs[i]) < unsigned(kv.max_seqs);
    }
#pragma unroll 1
    for (int g = tid; g < ng; g += kPlan) {
        groups = groups && 0 <= b.cu_group[g] && b.cu_group[g] <= b.cu_group[g + 1] && b.cu_group[g + 1] <= b.n;
        used[g] = INT_MAX;
        alone[g] = 0;
    }
    if (!order || !groups || !known) atomicMin(kv.status, SIM_E_INVAL);
    order = __syncthreads_and(order);
    groups = __syncthreads_and(groups);
    if (ng > 0) {
#pragma unroll 1
        for (int i0 = 0; i0 < b.n; i0 += kPlan) {  // the least number of pages of each group, the sum of its tile rows
            const int i = i0 + tid, g = i < b.n ? group_of(b, i) : -1, v = g < 0 ? INT_MAX : p.same[i];
            const int t = g < 0 ? 0 : tile_rows(entry_at(kv, b, i).t * G);
            int same_group;
            __match_all_sync(FULL, g, &same_group);
            if (same_group) {
                const int least = __reduce_min_sync(FULL, v), all = __reduce_add_sync(FULL, t);
                if (g >= 0 && (tid & 31) == 0) {
                    atomicMin(&used[g], least);
                    atomicAdd(&alone[g], all);
                }
            } else if (g >= 0) {
                atomicMin(&used[g], v);
                atomicAdd(&alone[g], t);
            }
        }
        __syncthreads();
    }
    if (ng > 0) {  // share where that saves time: in the group, and in all
        int64_t net = 0;
#pragma unroll 1
        for (int g = tid; g < ng; g += kPlan) {
            const int a = order && groups ? b.cu_group[g] : 0, z = order && groups ? b.cu_group[g + 1] : 0;
            KvSource x = {};
            x.prefix = -1;
            if (a < z) {
                x.q0 = b.cu_q[a];
                const int rows = (b.cu_q[z] - x.q0) * G, found = used[g] != INT_MAX ? used[g] : 0;
                const int64_t saves = int64_t(found * P / kTileKeys) * (alone[g] - tile_rows(rows)) - kShareItem - int64_t(rows) * kShareRows / 32;
                if (saves > 0) {
                    net += saves;
                    x.rows = rows;
                    x.seq = b.seqs[a];
                    x.kv1 = found * P;
                    x.pos0 = 1 << 30;
                }
            }
            source[g] = x;
        }
        if (net > 0) atomicAdd(&saved, static_cast<unsigned long long>(net));
        __syncthreads();
        if (int64_t(saved) * kv.n_kv_heads < int64_t(kShareOnce) * kv_blocks(sms, 1)) {
#pragma unroll 1
            for (int g = tid; g < ng; g += kPlan) source[g].rows = source[g].kv1 = 0;
            __syncthreads();
        }
    }
    int64_t sum = 0;  // heavy items, light ones above
#pragma unroll 1
    for (int s0 = 0; s0 < n_src; s0 += kPlan) {
        const int s = s0 + tid;
        KvSource x = {};
        if (s < ng) {
            x = source[s];
        } else if (s < n_src) {
            const Entry e = entry_at(kv, b, s - ng);
            const int g = group_of(b, s - ng), shared = g < 0 ? 0 : source[g].kv1;
            x.q0 = e.a;
            x.rows = order ? e.t * G : 0;
            x.seq = e.seq;
            x.kv0 = shared;
            x.kv1 = e.len;
            x.pos0 = e.len - e.t;
            x.prefix = shared > 0 ? g : -1;
            x.blind = e.len < e.t;
        }
        Two total;
        const int64_t before = sum + plan_scan<kPlan / 32>({int64_t(light_items(x.rows, only)) << 32 | heavy_items(x.rows, only), 0}, sums, total).a;
        sum += total.a;
        if (s < n_src) {
            x.heavy0 = first0[s] = int(before & 0xffffffff);
            x.light0 = first1[s] = int(before >> 32);
            x.n_heavy = heavy_items(x.rows, only);
            source[s] = x;
            if (FEW) p.source[s] = x;
            if (x.rows > 0 && (x.prefix >= 0 || x.blind)) p.join[atomicAdd(&counts[2], 1)] = s - ng;
        }
    }
    const int n_heavy = int(sum & 0xffffffff), n_light = int(sum >> 32);
    if (tid == 0) {
        first0[n_src] = p.hdr[0] = n_heavy;
        first1[n_src] = p.hdr[16] = n_light;
        p.hdr[1] = order;
    }
    __syncthreads();
#pragma unroll 1
    for (int light = 0; light < 2; ++light) {
        const int n_items = light ? n_light : n_heavy, blocks = kv_blocks(sms, light);
        const int32_t *first = light ? first1 : first0;
        KvItem *const items = light ? p.items[1] : p.items[0];
        Two done = {0, 0};  // spans, rows
#pragma unroll 1
        for (int k0 = 0; k0 < n_items; k0 += kPlan) {
            const int k = k0 + tid;
            KvItem it = {};
            int of = -1;  // source whose (first) light item this is
            if (k < n_items) {
                const int s = last_at_most(first, n_src, k);
                const KvSource x = source[s];
                it.row0 = only ? (k - x.light0) * kLightRows : (light ? x.n_heavy : k - x.heavy0) * kAttRows;
                it.rows = min(x.rows - it.row0, kv_rows(light));
                it.q0 = x.q0;
                it.seq = x.seq;
                it.kv0 = x.kv0;
                it.pos0 = x.pos0;
                it.kv1 = min(x.kv1, x.pos0 + (it.row0 + it.rows - 1) / G + 1);
                it.partial = s < ng || x.prefix >= 0;
                it.tiles = ceil_div(max(it.kv1 - it.kv0, 0), kTileKeys);
                if (light && it.row0 == x.n_heavy * kAttRows) of = s;
            }
            Two total;
            const Two before = plan_scan<kPlan / 32>({int64_t(kv_span(it.tiles, light)) * kv.n_kv_heads, int64_t(it.rows) * kv.n_kv_heads}, sums, total);
            it.unit = done.a + before.a;
            it.row_off = done.b + before.b;
            done = {done.a + total.a, done.b + total.b};
            if (k < n_items) {
                items[k] = it;
                if (FEW) {
                    few_units[k] = it.unit;
                    few_tiles[k] = it.partial ? -1 : it.tiles;
                }
                if (of >= 0) {
                    KvSource *const to = p.source + of;
                    to->tiles = it.tiles;
                    to->unit = it.unit;
                    to->row_off = it.row_off;
                }
            }
        }
        const Share share(done.a, blocks);
        if (tid == 0) {
            int32_t *h = p.hdr + 16 * light;
            *reinterpret_cast<int64_t *>(h + 2) = done.a;
            *reinterpret_cast<int64_t *>(h + 4) = share.each;
            h[6] = share.rest;
            if (!light) *reinterpret_cast<int64_t *>(p.hdr + 24) = done.b;
        }
        __syncthreads();
        if (n_items == 0) continue;
        const int64_t base = list_base(p, light, sms);
#pragma unroll 1
        for (int c = tid; c < blocks; c += kPlan) {
            const int64_t u = share.at(c);
            int k;
            if (FEW) {
                k = last_at_most(few_units, n_items, u);
            } else {
                int lo = 0, hi = n_items;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (items[mid].unit <= u) lo = mid;
                    else hi = mid;
                }
                k = lo;
            }
            (light ? p.start[1] : p.start[0])[c] = k;
            if (u < done.a && c > 0 && (!FEW || (few_tiles[k] > 0 && few_units[k] != u))) {
                const KvItem it = items[k];
                const int span = kv_span(it.tiles, light), h = span > 0 ? int(uint32_t(u - it.unit) / uint32_t(span)) : 0;
                const int64_t from = it.unit + int64_t(h) * span + kv_lead(light), before = share.at(c - 1);  // tile 0
                if (u > from && u < from + it.tiles && before <= from && !it.partial) {
                    KvCut cut;
                    cut.h = h;
                    const int c0 = share.of(from);
                    cut.n = share.of(from + it.tiles - 1) - c0 + 1;
                    cut.row = piece_row(it, cut.h, c0, base, light);
                    cut.q0 = it.q0;
                    cut.row0 = it.row0;
                    cut.rows = it.rows;
                    (light ? p.cut[1] : p.cut[0])[atomicAdd(&counts[light], 1)] = cut;
                }
            }
        }
        __syncthreads();
    }
    if (tid == 0) {
        p.hdr[7] = counts[0];
        p.hdr[23] = counts[1];
        p.hdr[17] = counts[2];
    }
}

// ---- k_combine ----------------------------------------------------------------------------------------------

// The partial results of one item and head: row `row` in the first of n pieces of blocks c0, c0 + 1, ..
struct Pieces {
    int64_t row;
    int n, light;
    __device__ Pieces() : row(0), n(0), light(0) {}
    // unit, tiles, row_off, rows: of the item
    __device__ Pieces(const Share &share, int64_t base, int64_t unit, int tiles, int64_t row_off, int rows, int h, int light_) : row(0), n(0), light(light_) {
        if (tiles > 0) {
            const int64_t from = unit + int64_t(h) * kv_span(tiles, light) + kv_lead(light);
            const int c0 = share.of(from);
            n = share.of(from + tiles - 1) - c0 + 1;
            row = base + row_off + int64_t(h) * rows + int64_t(kv_rows(light)) * c0;
        }
    }
    // Row `in` of the item in piece i, -1 if there is none.
    __device__ int64_t at(int i, int in) const { return i >= 0 && i < n ? row + int64_t(kv_rows(light)) * i + in : -1; }
};

constexpr int kJoin = 128;      // threads
constexpr int kJoinRows = 8;    // rows of a block at a time, 16 lanes each: as many as a token has heads in a group, often
constexpr int kJoinHeavy = 16;  // blocks for each cut of a heavy item, of a light one
constexpr int kJoinLight = 4;

// Rows whose keys were divided among items or blocks, or that see none.  A chain of dependent loads bounds it, so it is
// kept short (what a row needs of its source lies in one record) and every row is a half warp's own: its lanes
// read the sums of 16 pieces at once and, four at a time without waiting in between, the pieces.  One wave of blocks
// goes over what there is to join: items without a prefix that blocks' stretches cut, then entries with a shared prefix
// and rows without keys, by kv head (`parts` blocks for each).  Loads of pieces that are not there are made all the same, from
// another piece's row, so that the four of a lane need not be told apart (64 rows in 38 pieces: 118 us the whole call either way).
// 18 us for 16384 rows with a prefix in 3 or 4 pieces and their own keys, 15 us for the cuts of 152 heavy stretches.
template <bool BF>
__global__ void __launch_bounds__(kJoin, 5) k_combine(const sim_kv kv, const sim_kv_batch b, const KvAttend a, int parts) {
    kv_wait_previous();
    const KvPlan plan = kv_plan(kv, b);
    const int H = kv.n_kv_heads, G = b.q_heads / H, D = kv.head_dim, sl = threadIdx.x & 15, sub = threadIdx.x >> 4;
    const unsigned mine = 0xffffu << (threadIdx.x & 16);
    const auto put = [&](int t, int qh, const float4 *v, float lse) {
        uint16_t *o = static_cast<uint16_t *>(a.out) + int64_t(t) * a.ot + int64_t(qh) * a.oh;
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (4 * (sl + 16 * q) < D) *reinterpret_cast<uint2 *>(o + 4 * (sl + 16 * q)) = make_uint2(pack<BF>(v[q].x, v[q].y), pack<BF>(v[q].z, v[q].w));
        if (sl == 0 && a.lse) a.lse[int64_t(t) * b.q_heads + qh] = lse;
    };
    const uint32_t heavy = uint32_t(plan.hdr[7]) * kJoinHeavy, cuts = heavy + uint32_t(plan.hdr[23]) * kJoinLight;
    const uint32_t all = cuts + uint32_t(plan.hdr[17]) * uint32_t(H) * uint32_t(parts);  // at most 2^30 and the cuts
    const Share share0(plan, 0), share1(plan, 1);
    const int per_item = kv_rows(kv_light_only(kv, b));
    const int64_t base1 = list_base(plan, 1, a.sms);
#pragma unroll 1
    for (uint32_t y = blockIdx.x; y < all; y += gridDim.x) {
        // rows z, z + step, .. below z1 of query tokens from q0 on, and kv head h
        Pieces first, own;
        KvSource x;
        int q0, h, z, z1, step;
        const bool by_cut = y < cuts;
        if (by_cut) {
            const bool light = y >= heavy;
            const uint32_t nth = light ? y - heavy : y, per = light ? kJoinLight : kJoinHeavy, c = nth / per;
            const KvCut cut = (light ? plan.cut[1] : plan.cut[0])[c];
            own.row = cut.row - cut.row0;
            own.n = cut.n;
            own.light = light;
            q0 = cut.q0;
            h = cut.h;
            z = cut.row0 + int(nth - c * per) * kJoinRows + sub;
            z1 = cut.row0 + cut.rows;
            step = kJoinRows * int(per);
        } else {
            const uint32_t pairs = uint32_t(plan.hdr[17]) * uint32_t(H), part = (y - cuts) / pairs, ih = (y - cuts) - part * pairs, i = ih / uint32_t(H);
            h = int(ih - i * H);
            x = plan.source[b.n_groups + plan.join[i]];
            q0 = x.q0;
            z = int(part) * kJoinRows + sub;
            z1 = x.rows;
            step = kJoinRows * parts;
        }
#pragma unroll 1
        for (; z < z1; z += step) {
            const int dt = a.group.div(z), t = q0 + dt, qh = h * G + z - dt * G;
            int in = z, pin = 0;
            if (!by_cut) {
                if (x.prefix < 0) {  // only rows of items without keys: the item's last row sees the most
                    const int end = min(z / per_item * per_item + per_item, x.rows);
                    if (min(x.kv1, x.pos0 + int(a.group.div(end - 1)) + 1) > 0) continue;
                } else {
                    const int nth = z / kAttRows;
                    in = z % kAttRows;
                    if (nth >= x.n_heavy) {
                        own = Pieces(share1, base1, x.unit, x.tiles, x.row_off, min(x.rows - nth * kAttRows, kAttRows), h, 1);
                    } else {
                        const KvItem it = plan.items[0][x.heavy0 + nth];
                        own = Pieces(share0, 0, it.unit, it.tiles, it.row_off, it.rows, h, 0);
                    }
                    const KvSource px = plan.source[x.prefix];
                    const int row = (q0 - px.q0) * G + z, pth = row / kAttRows;
                    pin = row % kAttRows;
                    if (pth >= px.n_heavy) {
                        first = Pieces(share1, base1, px.unit, px.tiles, px.row_off, min(px.rows - pth * kAttRows, kAttRows), h, 1);
                    } else {
                        const KvItem it = plan.items[0][px.heavy0 + pth];
                        first = Pieces(share0, 0, it.unit, it.tiles, it.row_off, it.rows, h, 0);
                    }
                }
            }
            const int n = first.n + own.n;
            float top = -INFINITY, total = 0.f;
            float4 acc[2] = {};
#pragma unroll 1
            for (int p0 = 0; p0 < n; p0 += 16) {
                const int p = p0 + sl;
                int64_t at = p < first.n ? first.at(p, pin) : own.at(p - first.n, in);
                const float s = at >= 0 ? __ldcg(a.part_lse + at) : -INFINITY;
                const int64_t some = __shfl_sync(mine, at, 0, 16);
                at = at >= 0 ? at : some;  // a piece that is not there: another, with weight 0
                float4 v[4][2];
                const auto fetch = [&](int i0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 *from = reinterpret_cast<const float4 *>(a.part + __shfl_sync(mine, at, i0 + e, 16) * D);
#pragma unroll
                        for (int q = 0; q < 2; ++q) v[e][q] = __ldcg(from + (4 * (sl + 16 * q) < D ? sl + 16 * q : 0));
                    }
                };
                fetch(0);  // on their way while the sums are waited for
                float up = s;
#pragma unroll
                for (int d = 8; d >= 1; d >>= 1) up = fmaxf(up, __shfl_xor_sync(mine, up, d));
                up = fmaxf(up, top);
                const float w = s == -INFINITY ? 0.f : ex2(s - up), f = top == -INFINITY ? 0.f : ex2(top - up);
                top = up;
                total *= f;
#pragma unroll
                for (int q = 0; q < 2; ++q) acc[q] = make_float4(acc[q].x * f, acc[q].y * f, acc[q].z * f, acc[q].w * f);
#pragma unroll 1
                for (int i0 = 0; i0 < min(16, n - p0); i0 += 4) {
                    if (i0 > 0) fetch(i0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float we = __shfl_sync(mine, w, i0 + e, 16);
                        total += we;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const float4 u = v[e][q];
                            acc[q] = we == 0.f ? acc[q] : make_float4(fmaf(u.x, we, acc[q].x), fmaf(u.y, we, acc[q].y), fmaf(u.z, we, acc[q].z), fmaf(u.w, we, acc[q].w));
                        }
                    }
                }
            }
            const float f = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (int q = 0; q < 2; ++q) acc[q] = make_float4(acc[q].x * f, acc[q].y * f, acc[q].z * f, acc[q].w * f);
            put(t, qh, acc, total == 0.f ? -INFINITY : (top + log2f(total)) * 0.69314718055994531f);
        }
    }
    // query tokens of no entry
    const bool order = b.n > 0 && plan.hdr[1];
    const int before = order ? b.cu_q[0] : b.n_q, after = order ? b.cu_q[b.n] : b.n_q;
    const uint32_t rest = uint32_t(before + b.n_q - after) * uint32_t(b.q_heads);  // at most 2^30
    const float4 zero[2] = {};
#pragma unroll 1
    for (uint32_t x = blockIdx.x * kJoinRows + sub; x < rest; x += gridDim.x * kJoinRows) {
        const int e = int(x / uint32_t(b.q_heads));
        put(e < before ? e : e - before + after, int(x) - e * b.q_heads, zero, -INFINITY);
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

}  // namespace

bool kv_encode_map(const sim_kv &kv, CUtensorMap *map, int rank, const void *at, const uint64_t *dim, const uint64_t *stride, const uint32_t *box) {
    const EncodeFn encode = encode_fn();
    const cuuint32_t step[5] = {1, 1, 1, 1, 1};
    cuuint64_t dims[5], strides[5];
    for (int i = 0; i < rank; ++i) dims[i] = dim[i];
    for (int i = 0; i + 1 < rank; ++i) strides[i] = stride[i];
    return encode && encode(map, kv.dtype == SIM_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void *>(at), dims, strides,
                            box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_kv_plan(const sim_kv &kv, const sim_kv_batch &b, cudaStream_t st) {
    if (b.n_groups > 0) {
        cudaError_t e = launch_chained(k_plan_shared, std::max((b.n + 7) / 8, 1), 256, 0, st, kv, b);
        if (e != cudaSuccess) return e;
    }
    const KvPlan p = kv_plan(kv, b);
    const bool few = b.n_groups + b.n <= kFewSources && int64_t(p.max_heavy) <= kFewItems;  // at most one light item a source
    return launch_chained(few ? k_plan_items<true> : k_plan_items<false>, 1, few ? 512 : 1024, 0, st, kv, b, kv_sm_count());
}

cudaError_t launch_kv_attend(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    if (!encode_fn()) return cudaErrorNotSupported;
    KvMaps maps = {};
    for (int v = 0; v < 2; ++v) {
        uint16_t *at = static_cast<uint16_t *>(kv.pool) + a.layer * kv_layer_elems(kv) + v * (kv_layer_elems(kv) / 2);
        const uint64_t dim[4] = {uint64_t(kv.head_dim), uint64_t(kv.page_size), uint64_t(kv.n_kv_heads), uint64_t(kv.n_pages)};
        const uint64_t stride[3] = {uint64_t(kv.head_dim) * 2, uint64_t(kv.head_dim) * 2 * kv.page_size, uint64_t(kv_page_bytes(kv))};
        const uint32_t box[4] = {64, uint32_t(kv.page_size), 1, 1};
        if (!kv_encode_map(kv, v ? &maps.values : &maps.keys, 4, at, dim, stride, box)) return cudaErrorInvalidValue;
    }
    const int64_t rows = int64_t(b.n_q) * b.q_heads;
    cudaError_t e = cudaSuccess;
    if (!kv_light_only(kv, b)) e = launch_kv_heavy(kv, b, a, maps, st);
    if (e == cudaSuccess) e = launch_kv_light(kv, b, a, maps, st);
    if (e != cudaSuccess) return e;
    // blocks for an entry and head: for twice the rows that they have on average
    const int64_t parts = std::min<int64_t>(std::max<int64_t>((2 * rows / kv.n_kv_heads / std::max(b.n, 1) + kJoinRows - 1) / kJoinRows, 1), 16);
    const int blocks = int(std::min<int64_t>(rows, int64_t(a.sms) * 5));
    return launch_chained(kv.dtype == SIM_KV_BF16 ? k_combine<true> : k_combine<false>, blocks, kJoin, 0, st, kv, b, a, int(parts));
}

}  // namespace simgb
