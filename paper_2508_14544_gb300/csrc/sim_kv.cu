// Pages of the key/value cache (include/sim_kv.h): giving out, sharing, copying, freeing, compacting, writing.
//
// The metadata is small and its work serial in places (which page is the k-th free one), so a call is bound by
// launches and by the latency of dependent loads, not by bytes; what moves keys and values is bound by HBM:
//   k_extend   - one block.  Entry i needs n_i = ceil((L + new) / P) - ceil(L / P) pages, one more where its last
//                page is shared and has room; an exclusive scan over the entries places each entry's pages in the list of
//                the sum(n_i) lowest free ones, which 32 warps find by counting zeros of `ref` in a run of pages each,
//                a scan over the warps and a second walk.  Nothing is changed before the sum is known to fit.  6 us for
//                40 entries, 10 us for 250 entries and 16000 new pages, most of it chains of loads from L2.
//   k_move     - puts the pages into the tables, and makes the slots of the new tokens and the copies that k_extend
//                listed, whole pages of all layers.  Every byte read once and written once, 16 bytes a load, eight in
//                flight a thread, past L1 and L2: 80 us for 0.53 GB moved, 6.6 TB/s.
//   k_free, k_fork - a warp for each entry; `ref` changes by atomics whose order does not matter.  7 and 6 us for 256 entries.
//   k_compact  - one block: with N pages in use, the i-th used page at or above N goes to the i-th free one below N.  6 us for
//                4600 pages; k_compact_move makes the copies, 78 us for 0.52 GB, 6.6 TB/s.
//   k_write    - a thread for each 16 bytes of a token's keys and of its values, both loads before both stores, no thread with
//                more than one of each and stores that L2 need not keep: 285 us for 2.02 GB, 7.1 TB/s, the last writes still in
//                L2 (26 us more with 16 blocks per SM that stay).  Sources that are not 16-byte aligned are read 2 bytes at a time, as they must be.
#include <algorithm>
#include <climits>

#include "sim.h"
#include "sim_kv_internal.h"

namespace simgb {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int kMeta = 1024;   // threads of the one-block kernels
constexpr int kMove = 256;    // threads of the moving kernels
constexpr int kUnroll = 8;    // 16-byte loads in flight per thread
constexpr int kChunk = kMove * kUnroll * 16;
// Blocks per SM of the moving kernels, many more than fit: blocks that come as others end keep HBM busier than as many as fit,
// each with its share (0.53 GB, the free list included: 108 us with 4, 106 with 8, 103 with 32).
constexpr int kMoveWaves = 32;
// Sums over the entries of a call: pages in the low bits (at most n_pages + 1 <= 2^28 + 1 counted for an entry, 2^17
// entries), copies of shared pages above.
constexpr int kCowShift = 46;

__device__ __forceinline__ void report(const sim_kv &kv, int code) { atomicMin(kv.status, code); }

__device__ __forceinline__ int pages_of(int tokens, int P) { return (tokens + P - 1) / P; }

// Exclusive prefix sum of one value per thread of a block of kMeta threads, and the total.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t *sums, uint64_t &total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    uint64_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint64_t y = __shfl_up_sync(FULL, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) sums[w] = x;
    __syncthreads();
    if (w == 0) {
        uint64_t s = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint64_t y = __shfl_up_sync(FULL, s, d);
            if (lane >= d) s += y;
        }
        sums[lane] = s;
    }
    __syncthreads();
    total = sums[31];
    const uint64_t before = (w ? sums[w - 1] : 0) + x - v;
    __syncthreads();
    return before;
}

// Marks the sequences that the call names, and those named more than once, in two bit sets of max_seqs bits.
__device__ __forceinline__ void mark_named(uint32_t *once, uint32_t *twice, int words, int max_seqs, int n, const int32_t *seqs) {
    for (int i = threadIdx.x; i < 2 * words; i += blockDim.x) once[i] = 0;  // twice follows once
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int s = seqs[i];
        if (unsigned(s) < unsigned(max_seqs)) {
            const uint32_t bit = 1u << (s & 31);
            if (atomicOr(&once[s >> 5], bit) & bit) atomicOr(&twice[s >> 5], bit);
        }
    }
    __syncthreads();
}
__device__ __forceinline__ bool has(const uint32_t *set, int s) { return set[s >> 5] >> (s & 31) & 1; }

// The four words of `ref` at page p (a multiple of 4); pages past the end count as in use.
__device__ __forceinline__ int4 refs_at(const sim_kv &kv, int64_t p) {
    if (p + 4 <= kv.n_pages) return *reinterpret_cast<const int4 *>(kv.ref + p);
    int4 r = make_int4(1, 1, 1, 1);
    if (p < kv.n_pages) r.x = kv.ref[p];
    if (p + 1 < kv.n_pages) r.y = kv.ref[p + 1];
    if (p + 2 < kv.n_pages) r.z = kv.ref[p + 2];
    return r;
}
__device__ __forceinline__ int zeros(int4 r) { return (r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0); }

__device__ __forceinline__ int warp_sum(int v) { return __reduce_add_sync(FULL, v); }
__device__ __forceinline__ int warp_excl(int v) {
    const int lane = threadIdx.x & 31;
    int x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(FULL, x, d);
        if (lane >= d) x += y;
    }
    return x - v;
}

// Each of the 32 warps owns the pages [first, last): its free pages, and those of the warps before it.
struct FreeRun {
    int64_t first, last;
    int before, total;
};
__device__ __forceinline__ FreeRun count_free(const sim_kv &kv, uint64_t *sums) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t span = ((int64_t(kv.n_pages) + 31) / 32 + 127) / 128 * 128;
    FreeRun f;
    f.first = span * w;
    f.last = min(span * (w + 1), int64_t(kv.n_pages));
    int c = 0;
#pragma unroll 4
    for (int64_t p = f.first + 4 * lane; p < f.last; p += 128) c += zeros(refs_at(kv, p));
    c = warp_sum(c);
    uint64_t total;
    const uint64_t before = block_scan(lane == 0 ? uint64_t(c) : 0, sums, total);
    f.before = int(__shfl_sync(FULL, before, 0));
    f.total = int(total);
    return f;
}

// COPY: entry i makes seqs[i] a copy of src[i]; otherwise it gets cu[i + 1] - cu[i] new tokens.
template <bool COPY>
__global__ void __launch_bounds__(kMeta) k_extend(const sim_kv kv, int n, const int32_t *__restrict__ seqs,
                                                  const int32_t *__restrict__ cu, int n_new, const int32_t *__restrict__ src) {
    extern __shared__ uint32_t sets[];
    __shared__ uint64_t sums[32];
    kv_wait_previous();
    const KvScratch sc = kv_scratch(kv);
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, P = kv.page_size, words = (kv.max_seqs + 31) / 32;
    uint32_t *once = sets, *twice = sets + words;
    mark_named(once, twice, words, kv.max_seqs, n, seqs);
    uint64_t sum = 0;
    bool bad = false, order = true;  // an entry to leave out; offsets in order
    for (int i0 = 0; i0 < n; i0 += kMeta) {
        const int i = i0 + tid;
        int need = -1, cow = 0;
        if (i < n) {
            const int s = seqs[i];
            bool ok = unsigned(s) < unsigned(kv.max_seqs) && !has(twice, s);
            if (ok) {
                const int L = kv.length[s];
                if (COPY) {
                    const int o = src[i];
                    ok = L == 0 && unsigned(o) < unsigned(kv.max_seqs) && !has(once, o);
                    if (ok) need = min(pages_of(kv.length[o], P), kv.max_pages);
                } else {
                    const int a = cu[i], b = cu[i + 1];
                    ok = 0 <= a && a <= b && b <= n_new && int64_t(L) + (b - a) <= int64_t(kv.max_pages) * P;
                    if (ok) {
                        const int have = pages_of(L, P);
                        need = pages_of(L + (b - a), P) - have;
                        if (b > a && L % P != 0) {
                            const int old = kv.table[int64_t(s) * kv.max_pages + have - 1];
                            cow = unsigned(old) < unsigned(kv.n_pages) && kv.ref[old] > 1;
                            need += cow;
                        }
                    }
                }
            }
            bad |= !ok;
            if (!COPY) order = order && 0 <= cu[i] && cu[i] <= cu[i + 1] && cu[i + 1] <= n_new;
        }
        uint64_t total;
        const uint64_t before = sum + block_scan(need > 0 ? uint64_t(min(need, kv.n_pages + 1)) | uint64_t(cow) << kCowShift : 0, sums, total);
        sum += total;
        if (i < n) {
            const int64_t nth = before & ((uint64_t(1) << kCowShift) - 1), copy = before >> kCowShift;
            sc.base[i] = int(min(nth, int64_t(kv.n_pages)));
            sc.need[i] = need < 0 ? -1 : need << 1 | cow;
            if (!COPY && need >= 0) sc.len[i] = kv.length[seqs[i]];
            if (!COPY && cow && copy < kv.n_pages) {  // the copy's source; its destination is known once the pages are
                const int s = seqs[i];
                sc.src[copy] = kv.table[int64_t(s) * kv.max_pages + pages_of(kv.length[s], P) - 1];
                sc.dst[copy] = sc.base[i];
            }
        }
    }
    if (bad || !order) report(kv, SIM_E_INVAL);
    order = __syncthreads_and(order);
    const int64_t all_need = sum & ((uint64_t(1) << kCowShift) - 1);
    const int n_need = int(min(all_need, int64_t(kv.n_pages) + 1)), n_cow = int(sum >> kCowShift);
    if (n_need > 0 || !order) {
        const FreeRun f = count_free(kv, sums);
        const bool fits = n_need <= f.total;
        if (!fits || !order) {  // as a whole: no entry is left half done
            if (tid == 0) {
                if (!fits && order) report(kv, SIM_E_NOMEM);
                sc.hdr[0] = 0;
            }
            for (int i = tid; i < n; i += kMeta) sc.need[i] = -1;
            return;
        }
        int at = f.before;
        for (int64_t p0 = f.first; p0 < f.last && at < n_need; p0 += 128) {
            const int4 r = refs_at(kv, p0 + 4 * lane);
            const int c = zeros(r);
            int k = at + warp_excl(c);
            const int p = int(p0) + 4 * lane;
            if (r.x == 0 && k < n_need) sc.free[k] = p;
            k += r.x == 0;
            if (r.y == 0 && k < n_need) sc.free[k] = p + 1;
            k += r.y == 0;
            if (r.z == 0 && k < n_need) sc.free[k] = p + 2;
            k += r.z == 0;
            if (r.w == 0 && k < n_need) sc.free[k] = p + 3;
            at += warp_sum(c);
        }
        __syncthreads();
    }
    if (tid == 0) sc.hdr[0] = COPY ? n_need : n_cow;
    if constexpr (!COPY) {  // k_move does the rest
        for (int c = tid; c < n_cow; c += kMeta) sc.dst[c] = sc.free[sc.dst[c]];
    } else {
        for (int i = w; i < n; i += kMeta / 32) {
            const int need = sc.need[i] >> 1, base = sc.base[i];
            if (need < 0) continue;
            const int s = seqs[i];
            int32_t *row = kv.table + int64_t(s) * kv.max_pages;
            const int32_t *from = kv.table + int64_t(src[i]) * kv.max_pages;
            for (int j = lane; j < need; j += 32) {
                const int page = sc.free[base + j];
                row[j] = page;
                kv.ref[page] = 1;
                sc.src[base + j] = from[j];
                sc.dst[base + j] = page;
            }
            __syncwarp();
            if (lane == 0) kv.length[s] = kv.length[src[i]];
        }
    }
}

// Copies whole pages, chunk by chunk over the grid.  No page is both a source and a destination.
__device__ __forceinline__ void move_pages(const sim_kv &kv, int count, const int32_t *src, const int32_t *dst) {
    const int64_t bytes = kv_page_bytes(kv), per = (bytes + kChunk - 1) / kChunk, all = per * count;
    for (int64_t c = blockIdx.x; c < all; c += gridDim.x) {
        const int m = int(c / per), a = src[m], b = dst[m];
        if (unsigned(a) >= unsigned(kv.n_pages) || unsigned(b) >= unsigned(kv.n_pages)) continue;
        const int64_t off = (c - m * per) * kChunk;
        const uint4 *from = reinterpret_cast<const uint4 *>(static_cast<const char *>(kv.pool) + a * bytes + off);
        uint4 *to = reinterpret_cast<uint4 *>(static_cast<char *>(kv.pool) + b * bytes + off);
        const int vecs = int(min(int64_t(kChunk), bytes - off) / 16);
        uint4 x[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
            if (threadIdx.x + k * kMove < vecs) x[k] = __ldcs(from + threadIdx.x + k * kMove);
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
            if (threadIdx.x + k * kMove < vecs) __stcs(to + threadIdx.x + k * kMove, x[k]);
    }
}

// Last index i in [0, n) with cu[i] <= t, or -1.
__device__ __forceinline__ int entry_of(const int32_t *cu, int n, int t) {
    int lo = -1, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kMove) k_move(const sim_kv kv, int n, const int32_t *__restrict__ seqs,
                                                const int32_t *__restrict__ cu, int n_new, int64_t *__restrict__ slots) {
    kv_wait_previous();
    const KvScratch sc = kv_scratch(kv);
    const int P = kv.page_size, lane = threadIdx.x & 31, first = blockIdx.x * kMove + threadIdx.x, all = gridDim.x * kMove;
    if (cu) {
        // a warp for each entry: its new pages, from the one that replaces a shared last page on
        for (int i = first >> 5; i < n; i += all >> 5) {
            const int need = sc.need[i] >> 1, cow = sc.need[i] & 1, base = sc.base[i];
            if (need < 0) continue;
            const int s = seqs[i], L = sc.len[i];
            int32_t *row = kv.table + int64_t(s) * kv.max_pages + pages_of(L, P) - cow;
            for (int j = lane; j < need; j += 32) {
                const int page = sc.free[base + j];
                row[j] = page;
                kv.ref[page] = 1;
            }
            if (lane == 0) kv.length[s] = L + (cu[i + 1] - cu[i]);
        }
        for (int c = first; c < sc.hdr[0]; c += all) atomicSub(&kv.ref[sc.src[c]], 1);
        for (int64_t t = first; t < n_new; t += all) {
            const int i = entry_of(cu, n, int(t));
            int64_t slot = -1;
            if (i >= 0 && t < cu[i + 1] && sc.need[i] >= 0) {
                // of pages that were there only the table knows, of new ones the list
                const int L = sc.len[i], pos = L + int(t) - cu[i], nth = pos / P - (pages_of(L, P) - (sc.need[i] & 1));
                const int page = nth >= 0 ? sc.free[sc.base[i] + nth] : kv.table[int64_t(seqs[i]) * kv.max_pages + pos / P];
                slot = int64_t(page) * P + pos % P;
            }
            slots[t] = slot;
        }
    }
    move_pages(kv, sc.hdr[0], sc.src, sc.dst);
}

__global__ void __launch_bounds__(kMove) k_free(const sim_kv kv, int n, const int32_t *__restrict__ seqs,
                                                const int32_t *__restrict__ keep) {
    extern __shared__ uint32_t sets[];
    kv_wait_previous();
    const int words = (kv.max_seqs + 31) / 32, P = kv.page_size, lane = threadIdx.x & 31;
    mark_named(sets, sets + words, words, kv.max_seqs, n, seqs);
    for (int i = (blockIdx.x * kMove + threadIdx.x) >> 5; i < n; i += gridDim.x * kMove >> 5) {
        const int s = seqs[i], want = keep ? keep[i] : 0;
        if (unsigned(s) >= unsigned(kv.max_seqs) || has(sets + words, s) || want < 0) {
            if (lane == 0) report(kv, SIM_E_INVAL);
            continue;
        }
        const int L = kv.length[s], left = min(want, L), have = min(pages_of(L, P), kv.max_pages);
        int32_t *row = kv.table + int64_t(s) * kv.max_pages;
        for (int j = pages_of(left, P) + lane; j < have; j += 32) {
            const int page = row[j];
            row[j] = -1;
            if (unsigned(page) < unsigned(kv.n_pages)) atomicSub(&kv.ref[page], 1);
        }
        __syncwarp();
        if (lane == 0) kv.length[s] = left;
    }
}

__global__ void __launch_bounds__(kMove) k_fork(const sim_kv kv, int n, const int32_t *__restrict__ src,
                                                const int32_t *__restrict__ dst, const int32_t *__restrict__ tokens) {
    extern __shared__ uint32_t sets[];
    kv_wait_previous();
    const int words = (kv.max_seqs + 31) / 32, P = kv.page_size, lane = threadIdx.x & 31;
    mark_named(sets, sets + words, words, kv.max_seqs, n, dst);
    for (int i = (blockIdx.x * kMove + threadIdx.x) >> 5; i < n; i += gridDim.x * kMove >> 5) {
        const int s = src[i], d = dst[i];
        bool ok = unsigned(s) < unsigned(kv.max_seqs) && unsigned(d) < unsigned(kv.max_seqs);
        ok = ok && !has(sets + words, d) && !has(sets, s) && kv.length[d] == 0;
        const int L = ok ? kv.length[s] : 0, take = tokens ? tokens[i] : L;
        if (!ok || take < 0 || take > L) {
            if (lane == 0) report(kv, SIM_E_INVAL);
            continue;
        }
        const int32_t *from = kv.table + int64_t(s) * kv.max_pages;
        int32_t *to = kv.table + int64_t(d) * kv.max_pages;
        for (int j = lane; j < min(pages_of(take, P), kv.max_pages); j += 32) {
            const int page = from[j];
            to[j] = page;
            if (unsigned(page) < unsigned(kv.n_pages)) atomicAdd(&kv.ref[page], 1);
        }
        __syncwarp();
        if (lane == 0) kv.length[d] = take;
    }
}

__global__ void __launch_bounds__(kMeta) k_compact(const sim_kv kv, int32_t *__restrict__ to) {
    __shared__ uint64_t sums[32];
    __shared__ int below;
    kv_wait_previous();
    const KvScratch sc = kv_scratch(kv);
    const int lane = threadIdx.x & 31;
    const FreeRun f = count_free(kv, sums);
    const int used = kv.n_pages - f.total;  // pages below this number stay or are filled
    // free pages below `used`: as many as used pages at or above it
    const auto walk = [&](auto &&visit) {
        int at = f.before;  // free pages before the one visited
        for (int64_t p0 = f.first; p0 < f.last; p0 += 128) {
            const int4 r = refs_at(kv, p0 + 4 * lane);
            const int c = zeros(r), p = int(p0) + 4 * lane;
            int k = at + warp_excl(c);
            visit(p, r.x, k);
            k += r.x == 0;
            visit(p + 1, r.y, k);
            k += r.y == 0;
            visit(p + 2, r.z, k);
            k += r.z == 0;
            visit(p + 3, r.w, k);
            at += warp_sum(c);
        }
    };
    if (threadIdx.x == 0) below = f.total;  // no free page at or above `used`
    __syncthreads();
    walk([&](int p, int, int k) {
        if (p == used) below = k;
    });
    __syncthreads();
    const int moves = below;
    walk([&](int p, int r, int k) {
        if (p >= kv.n_pages) return;
        if (r == 0) {
            to[p] = -1;
            if (p < used) sc.dst[k] = p;
        } else if (p < used) {
            to[p] = p;
        } else {
            sc.src[(p - used) - (k - moves)] = p;
        }
    });
    __syncthreads();
    for (int m = threadIdx.x; m < moves; m += kMeta) to[sc.src[m]] = sc.dst[m];
    if (threadIdx.x == 0) sc.hdr[0] = moves;
}

// Moves the pages that k_compact listed, and rewrites `ref` and the tables.
__global__ void __launch_bounds__(kMove) k_compact_move(const sim_kv kv, const int32_t *__restrict__ to) {
    kv_wait_previous();
    const KvScratch sc = kv_scratch(kv);
    const int moves = sc.hdr[0], first = blockIdx.x * kMove + threadIdx.x, all = gridDim.x * kMove;
    for (int m = first; m < moves; m += all) {
        kv.ref[sc.dst[m]] = kv.ref[sc.src[m]];
        kv.ref[sc.src[m]] = 0;
    }
    if (moves > 0)
        for (int s = first >> 5; s < kv.max_seqs; s += all >> 5) {
            const int have = min(pages_of(kv.length[s], kv.page_size), kv.max_pages);
            int32_t *row = kv.table + int64_t(s) * kv.max_pages;
            for (int j = threadIdx.x & 31; j < have; j += 32) {
                const int page = row[j];
                if (unsigned(page) < unsigned(kv.n_pages)) row[j] = to[page];
            }
        }
    move_pages(kv, moves, sc.src, sc.dst);
}

// A thread for each 16 bytes of a token's keys and of its values.  VEC: the sources are 16-byte aligned.
template <bool VEC>
__global__ void __launch_bounds__(kMove) k_write(const sim_kv kv, const KvWrite a, const FastDiv per_token, const FastDiv per_head) {
    kv_wait_previous();
    const int P = kv.page_size, D = kv.head_dim, shift = __ffs(P) - 1;
    const int64_t all = int64_t(a.n_new) * per_token.d, values = kv_layer_elems(kv) / 2;
    uint16_t *layer = static_cast<uint16_t *>(kv.pool) + a.layer * kv_layer_elems(kv);
    for (int64_t i0 = int64_t(blockIdx.x) * kMove; i0 < all; i0 += int64_t(gridDim.x) * kMove) {
        const int64_t i = i0 + threadIdx.x;
        if (i >= all) return;
        int t, r;
        if (all <= INT_MAX) {
            t = int(per_token.div(uint32_t(i)));
            r = int(i - int64_t(t) * per_token.d);
        } else {
            t = int(i / per_token.d);
            r = int(i % per_token.d);
        }
        const int h = int(per_head.div(uint32_t(r))), c = 8 * (r - h * int(per_head.d));
        const int64_t slot = a.slots[t], page = slot >> shift;
        if (slot < 0 || page >= kv.n_pages) continue;
        uint16_t *to = layer + page * (kv_page_bytes(kv) / 2) + (int64_t(h) * P + (slot & (P - 1))) * D + c;
        const uint16_t *k = static_cast<const uint16_t *>(a.k) + t * a.kt + h * a.kh + c;
        const uint16_t *v = static_cast<const uint16_t *>(a.v) + t * a.vt + h * a.vh + c;
        uint4 x, y;
        if (VEC) {
            x = __ldcs(reinterpret_cast<const uint4 *>(k));
            y = __ldcs(reinterpret_cast<const uint4 *>(v));
        } else {
            uint32_t xs[4], ys[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                xs[e] = k[2 * e] | uint32_t(k[2 * e + 1]) << 16;
                ys[e] = v[2 * e] | uint32_t(v[2 * e + 1]) << 16;
            }
            x = make_uint4(xs[0], xs[1], xs[2], xs[3]);
            y = make_uint4(ys[0], ys[1], ys[2], ys[3]);
        }
        __stcs(reinterpret_cast<uint4 *>(to), x);
        __stcs(reinterpret_cast<uint4 *>(to + values), y);
    }
}

size_t set_bytes(const sim_kv &kv) { return size_t(kv.max_seqs + 31) / 32 * 8; }

int blocks_for(int64_t items, int per_block, int per_sm) {
    return int(std::min<int64_t>(std::max<int64_t>(1, (items + per_block - 1) / per_block), int64_t(kv_sm_count()) * per_sm));
}

}  // namespace

int kv_sm_count() {
    static thread_local int dev_of = -1, count = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    if (dev != dev_of) {
        cudaDeviceGetAttribute(&count, cudaDevAttrMultiProcessorCount, dev);
        dev_of = dev;
    }
    return std::min(std::max(count, 1), kKvMaxSms);
}

cudaError_t launch_kv_extend(const sim_kv &kv, int32_t n, const int32_t *seqs, const int32_t *cu_new, int32_t n_new,
                             int64_t *slots, cudaStream_t st) {
    cudaError_t e = launch_chained(k_extend<false>, 1, kMeta, set_bytes(kv), st, kv, n, seqs, cu_new, n_new, static_cast<const int32_t *>(nullptr));
    if (e != cudaSuccess) return e;
    // at most one page copied for each entry
    const int64_t chunks = (kv_page_bytes(kv) + kChunk - 1) / kChunk * n;
    const int blocks = std::max(blocks_for(chunks, 1, kMoveWaves), blocks_for(n_new, kMove, 8));
    return launch_chained(k_move, blocks, kMove, 0, st, kv, n, seqs, cu_new, n_new, slots);
}

cudaError_t launch_kv_copy(const sim_kv &kv, int32_t n, const int32_t *src, const int32_t *dst, cudaStream_t st) {
    cudaError_t e = launch_chained(k_extend<true>, 1, kMeta, set_bytes(kv), st, kv, n, dst, static_cast<const int32_t *>(nullptr), 0, src);
    if (e != cudaSuccess) return e;
    return launch_chained(k_move, kv_sm_count() * kMoveWaves, kMove, 0, st, kv, n, dst, static_cast<const int32_t *>(nullptr), 0, static_cast<int64_t *>(nullptr));
}

cudaError_t launch_kv_fork(const sim_kv &kv, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *tokens, cudaStream_t st) {
    return launch_chained(k_fork, blocks_for(n, kMove / 32, 2), kMove, set_bytes(kv), st, kv, n, src, dst, tokens);
}

cudaError_t launch_kv_free(const sim_kv &kv, int32_t n, const int32_t *seqs, const int32_t *keep, cudaStream_t st) {
    return launch_chained(k_free, blocks_for(n, kMove / 32, 2), kMove, set_bytes(kv), st, kv, n, seqs, keep);
}

cudaError_t launch_kv_compact(const sim_kv &kv, int32_t *to, cudaStream_t st) {
    cudaError_t e = launch_chained(k_compact, 1, kMeta, 0, st, kv, to);
    if (e != cudaSuccess) return e;
    return launch_chained(k_compact_move, kv_sm_count() * kMoveWaves, kMove, 0, st, kv, static_cast<const int32_t *>(to));
}

cudaError_t launch_kv_write(const sim_kv &kv, const KvWrite &w, cudaStream_t st) {
    const int per_head = kv.head_dim / 8, per_token = per_head * kv.n_kv_heads;
    const auto aligned = [](const void *p, int64_t a, int64_t b) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && a % 8 == 0 && b % 8 == 0; };
    const bool vec = aligned(w.k, w.kt, w.kh) && aligned(w.v, w.vt, w.vh);
    const int blocks = blocks_for(int64_t(w.n_new) * per_token, kMove, 4096);
    return launch_chained(vec ? k_write<true> : k_write<false>, blocks, kMove, 0, st, kv, w, FastDiv(per_token), FastDiv(per_head));
}

}  // namespace simgb
