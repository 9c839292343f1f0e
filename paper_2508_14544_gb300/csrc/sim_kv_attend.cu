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
// The plan (k_plan_shared, k_plan_items, made once for all layers) lists the items.  Those of more than 128 rows
// are heavy, the others light: two kernels (sim_kv_heavy.cu, sim_kv_light.cu), because many rows want the tensor
// products fed and few rows want bytes in flight.  The tiles of all items and heads of a list lie on one line, and every block
// takes an equal stretch of it, so that work is even whatever the lengths; an item is split where two stretches meet, and
// k_combine joins the pieces.
#include <algorithm>

#include "sim_kv_attend.cuh"

namespace simgb {

namespace {

// ---- plan ---------------------------------------------------------------------------------------------------

constexpr int kPlan = 1024;
constexpr int kShareCost = 4;          // tiles of 128 rows that a second partial result of as many rows costs

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

__device__ __noinline__ int64_t plan_scan(int64_t v, int64_t *sums, int64_t &total) {
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
            const int64_t saved = int64_t(found * P / kv_tile(0)) * (p.alone[g] - tile_rows(rows));
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
        p.first[1][n_src] = p.hdr[16] = n_light;
        p.hdr[1] = order;
    }
    __syncthreads();
#pragma unroll 1
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
                it.tiles = ceil_div(max(it.kv1 - it.kv0, 0), kv_tile(light));
            }
            int64_t total;
            it.unit = units + plan_scan(int64_t(it.tiles) * kv.n_kv_heads, sums, total);
            units += total;
            it.row_off = list_rows + plan_scan(int64_t(it.rows) * kv.n_kv_heads, sums, total);
            list_rows += total;
            if (k < n_items) p.items[light][k] = it;
        }
        const int blocks = kv_blocks(sms, light);
        if (tid == 0) {
            int32_t *h = p.hdr + 16 * light;
            *reinterpret_cast<int64_t *>(h + 2) = units;
            *reinterpret_cast<int64_t *>(h + 4) = units / blocks;
            h[6] = int(units - units / blocks * blocks);
            if (!light) *reinterpret_cast<int64_t *>(p.hdr + 24) = list_rows;
        }
        __syncthreads();
        const Share share(p, light, sms);
        for (int c = tid; c < blocks; c += kPlan) {
            const int64_t u = share.at(c);
            int lo = 0, hi = n_items;  // the last item that begins at or before the block's stretch
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.items[light][mid].unit <= u) lo = mid;
                else hi = mid;
            }
            p.start[light][c] = lo;
            // an entry's item that has no prefix and is cut here for the first time: k_combine joins its pieces
            int cut_k = -1, cut_h = 0;
            if (u < units && c > 0) {
                const KvItem *it = p.items[light] + lo;
                cut_h = int(uint32_t(u - it->unit) / uint32_t(it->tiles));
                const int64_t from = it->unit + int64_t(cut_h) * it->tiles, before = share.at(c - 1);
                if (u > from && before <= from && before < u && !it->partial) cut_k = lo;
            }
            p.cut[light][2 * c] = cut_k;
            p.cut[light][2 * c + 1] = cut_h;
        }
    }
}

// ---- k_combine ----------------------------------------------------------------------------------------------

// The pieces of one item and head: those of blocks c0 .. c0 + n - 1 that have any of its tiles.
struct Pieces {
    Share share;
    int64_t row;
    int c0, n, rows;
    __device__ Pieces() : row(0), c0(0), n(0), rows(0) {}
    __device__ Pieces(const KvPlan &p, const KvItem &it, int h, int light, int sms) : share(p, light, sms), c0(0), n(0) {
        rows = light ? kAttRows / 2 : kAttRows;
        if (it.tiles > 0) {
            const int64_t from = it.unit + int64_t(h) * it.tiles;
            c0 = share.of(from);
            n = share.of(from + it.tiles - 1) - c0 + 1;
        }
        row = piece_row(it, h, c0, list_base(p, light, sms), light);
    }
    // Row `in` of the item in piece i, -1 if the block has none of its tiles (where there are fewer tiles than blocks).
    __device__ int64_t at(int i, int in) const {
        const bool some = share.each > 0 || share.at(c0 + i) < share.at(c0 + i + 1);
        return i >= 0 && i < n && some ? row + int64_t(rows) * i + in : -1;
    }
};

constexpr int kJoin = 256;     // threads
constexpr int kJoinHeavy = 4;  // blocks for each place where heavy items may be cut, light items
constexpr int kJoinLight = 2;

// Rows whose keys were divided among items or blocks, or that see none: a warp for each row, whose lanes first
// read the sums of 32 pieces and then, eight at a time without waiting in between, the pieces.  The first blocks go by
// the places where blocks' stretches meet, of which each cuts at most one item; the others by entry and kv head (`parts`
// blocks for each), for entries with a shared prefix and rows without keys.
template <bool BF>
__global__ void __launch_bounds__(kJoin, 4) k_combine(const sim_kv kv, const sim_kv_batch b, const KvAttend a, int parts) {
    kv_wait_previous();
    const KvPlan plan = kv_plan(kv, b);
    const int H = kv.n_kv_heads, G = b.q_heads / H, D = kv.head_dim, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int cols = 4 * lane < D ? lane : 0;  // this lane's four columns
    const auto put = [&](int t, int qh, float4 v, float lse) {
        if (4 * lane < D)
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + int64_t(t) * a.ot + int64_t(qh) * a.oh + 4 * lane) = make_uint2(pack<BF>(v.x, v.y), pack<BF>(v.z, v.w));
        if (lane == 0 && a.lse) a.lse[int64_t(t) * b.q_heads + qh] = lse;
    };
    const auto join = [&](const Pieces &first, int in, const Pieces &own, int r, int t, int qh) {
        const int n = first.n + own.n;
        float top = -INFINITY, total = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int p0 = 0; p0 < n; p0 += 32) {
            const int p = p0 + lane;
            const int64_t at = p < first.n ? first.at(p, in) : own.at(p - first.n, r);
            const float s = at >= 0 ? a.part_lse[at] : -INFINITY;
            float up = s;
#pragma unroll
            for (int d = 16; d >= 1; d >>= 1) up = fmaxf(up, __shfl_xor_sync(FULL, up, d));
            up = fmaxf(up, top);
            const float w = s == -INFINITY ? 0.f : ex2(s - up), f = top == -INFINITY ? 0.f : ex2(top - up);
            top = up;
            total *= f;
            acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
#pragma unroll 1
            for (int i0 = 0; i0 < min(32, n - p0); i0 += 8) {
                float4 v[8];  // a piece that is not there: row 0, with weight 0
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __ldcs(reinterpret_cast<const float4 *>(a.part + max(__shfl_sync(FULL, at, i0 + i), int64_t(0)) * D) + cols);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float wi = __shfl_sync(FULL, w, i0 + i);
                    total += wi;
                    acc = wi == 0.f ? acc : make_float4(fmaf(v[i].x, wi, acc.x), fmaf(v[i].y, wi, acc.y), fmaf(v[i].z, wi, acc.z), fmaf(v[i].w, wi, acc.w));
                }
            }
        }
        const float f = total == 0.f ? 0.f : 1.f / total;
        put(t, qh, make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f), total == 0.f ? -INFINITY : (top + log2f(total)) * 0.69314718055994531f);
    };
    const int heavy = kv_blocks(a.sms, 0) * kJoinHeavy, cuts = heavy + kv_blocks(a.sms, 1) * kJoinLight;
    const bool by_cut = int(blockIdx.x) < cuts;
    const int64_t all = by_cut ? cuts : int64_t(b.n) * H * parts + cuts;
#pragma unroll 1
    for (int64_t x = blockIdx.x; x < all; x += by_cut ? cuts : gridDim.x - cuts) {
        // rows z0, z0 + step, .. below z1 of the entry and head; a cut item's own rows
        int i, h, z0, z1, step;
        bool shared = false;
        if (by_cut) {
            const bool light = int(x) >= heavy;
            const int y = light ? int(x) - heavy : int(x), per = light ? kJoinLight : kJoinHeavy, c = y / per;
            const int k = plan.cut[light][2 * c];
            if (k < 0) break;
            h = plan.cut[light][2 * c + 1];
            const KvItem *it = plan.items[light] + k;
            i = it->entry;
            z0 = it->row0 + (y - c * per) * 8 + warp;
            z1 = it->row0 + it->rows;
            step = 8 * per;
        } else {
            const uint32_t y = uint32_t(x - cuts), ih = y / uint32_t(parts);
            i = int(ih / uint32_t(H));
            h = int(ih) - i * H;
            const Entry e = entry_at(kv, b, i);
            const int g = plan.group[i];
            shared = g >= 0 && plan.used[g] > 0;
            z0 = int(y - ih * parts) * 8 + warp;
            z1 = !plan.hdr[1] || (!shared && e.len >= e.t) ? 0 : e.t * G;  // none: k_attend has written these, or the cuts
            step = 8 * parts;
        }
        if (z0 >= z1) continue;
        const int q0 = b.cu_q[i], src = b.n_groups + i, heavy0 = plan.first[0][src], n_heavy = plan.first[0][src + 1] - heavy0, light0 = plan.first[1][src];
        const int g = shared ? plan.group[i] : 0, group_q0 = shared ? b.cu_q[b.cu_group[g]] : 0;
#pragma unroll 1
        for (int z = z0; z < z1; z += step) {
            const int dt = a.group.div(z), t = q0 + dt, qh = h * G + z - dt * G, nth = z / kAttRows;
            const bool light = nth >= n_heavy;
            const KvItem it = plan.items[light][light ? light0 : heavy0 + nth];
            if (!by_cut && !shared && it.tiles > 0) continue;  // only rows without keys
            Pieces first;
            int in = 0;
            if (shared) {
                const int row = (t - group_q0) * G + qh - h * G, pth = row / kAttRows, p0 = plan.first[0][g];
                const bool pl = pth >= plan.first[0][g + 1] - p0;
                first = Pieces(plan, plan.items[pl][pl ? plan.first[1][g] : p0 + pth], h, pl, a.sms);
                in = row % kAttRows;
            }
            join(first, in, Pieces(plan, it, h, light, a.sms), z % kAttRows, t, qh);
        }
    }
    // query tokens of no entry
    const bool order = b.n > 0 && plan.hdr[1];
    const int first = order ? b.cu_q[0] : b.n_q, last = order ? b.cu_q[b.n] : b.n_q;
    const uint32_t rest = uint32_t(first + b.n_q - last) * uint32_t(b.q_heads);  // at most 2^30
#pragma unroll 1
    for (uint32_t x = blockIdx.x * 8 + warp; x < rest; x += gridDim.x * 8) {
        const int i = int(x / uint32_t(b.q_heads));
        put(i < first ? i : i - first + last, int(x) - i * b.q_heads, make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY);
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

cudaError_t launch_kv_plan(const sim_kv &kv, const sim_kv_batch &b, cudaStream_t st) {
    if (b.n_groups > 0) {
        cudaError_t e = launch_chained(k_plan_shared, std::max((b.n + 7) / 8, 1), 256, 0, st, kv, b);
        if (e != cudaSuccess) return e;
    }
    return launch_chained(k_plan_items, 1, kPlan, 0, st, kv, b, kv_sm_count());
}

cudaError_t launch_kv_attend(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    const EncodeFn encode = encode_fn();
    if (!encode) return cudaErrorNotSupported;
    const auto encode_maps = [&](KvMaps &maps, int light) {
        for (int v = 0; v < 2; ++v) {
            uint16_t *at = static_cast<uint16_t *>(kv.pool) + a.layer * kv_layer_elems(kv) + v * (kv_layer_elems(kv) / 2);
            const cuuint64_t dim[4] = {cuuint64_t(kv.head_dim), cuuint64_t(kv.page_size), cuuint64_t(kv.n_kv_heads), cuuint64_t(kv.n_pages)};
            const cuuint64_t stride[3] = {cuuint64_t(kv.head_dim) * 2, cuuint64_t(kv.head_dim) * 2 * kv.page_size, cuuint64_t(kv_page_bytes(kv))};
            const cuuint32_t box[4] = {64, cuuint32_t(std::min(kv.page_size, kv_tile(light))), 1, 1}, step[4] = {1, 1, 1, 1};
            if (encode(v ? &maps.values : &maps.keys, kv.dtype == SIM_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, at, dim, stride,
                       box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
                return false;
        }
        return true;
    };
    KvMaps heavy, light;
    if (!encode_maps(light, 1)) return cudaErrorInvalidValue;
    heavy = light;
    if (kv.page_size > kv_tile(1) && !encode_maps(heavy, 0)) return cudaErrorInvalidValue;
    const int64_t rows = int64_t(b.n_q) * b.q_heads;
    cudaError_t e = cudaSuccess;
    if (rows / kv.n_kv_heads > kAttRows / 2) e = launch_kv_heavy(kv, b, a, heavy, st);  // fewer rows make no heavy item
    if (e == cudaSuccess) e = launch_kv_light(kv, b, a, light, st);
    if (e != cudaSuccess) return e;
    // as many blocks for an entry and head as its rows can use on average
    const int64_t parts = std::min<int64_t>(std::max<int64_t>(rows / kv.n_kv_heads / std::max(b.n, 1) / 8, 1), 16);
    const int cuts = kv_blocks(a.sms, 0) * kJoinHeavy + kv_blocks(a.sms, 1) * kJoinLight;
    const int blocks = cuts + int(std::min<int64_t>(std::max<int64_t>(b.n * int64_t(kv.n_kv_heads) * parts, 1), int64_t(a.sms) * 16));
    return launch_chained(kv.dtype == SIM_KV_BF16 ? k_combine<true> : k_combine<false>, blocks, kJoin, 0, st, kv, b, a, int(parts));
}

}  // namespace simgb
