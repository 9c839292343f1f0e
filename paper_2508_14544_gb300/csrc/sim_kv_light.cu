// Attention of light items (up to 32 query rows; see sim_kv_attend.cu): single tokens of one sequence and the
// few rows of small groups, bound by the bytes of the keys and values.
//
// Two blocks per SM, so that one loads while the other is between two items, and tiles of 64 keys, six (D > 64) or twelve of
// keys or values in flight in each: about 190 KB per SM.  Queries go to TMEM and are the products' first operand from
// there: no shared memory is spent on them.  Per tile: S = Q K^T (128 x 64 x D), P = exp2(c (S - m)) over S in TMEM,
// O += P V (128 x D x 64).  The products always have 128 rows, of which few are in use: the tensor unit has the time.
// Every row lies in TMEM four times, each copy with its own quarter of a tile's keys, so that
// the four warps of the softmax share few rows; the copies are joined at the end of the item.
#include "sim_kv_attend.cuh"

namespace simgb {

namespace {

template <int DP>
struct Shape {
    static constexpr int kThreads = 192;             // four softmax warps, one loads, one issues
    static constexpr int kTile = DP * 128;           // bytes of 64 keys or values
    static constexpr int kHalf = 8192;               // 64 rows of 64 columns
    static constexpr int kSlots = 98304 / kTile;
    static constexpr int kTmem = 256, kColQ = 64, kColO = 128;  // S / P below
    static constexpr int kOffStage = kSlots * kTile;
    static constexpr int kJoinStage = 2560;          // floats: 4 copies of 32 rows x (16 + 4), or of fewer and longer ones
    static constexpr int kOffStat = kOffStage + kJoinStage * 4;
    static constexpr int kOffAgain = kOffStat + 2 * 128 * 8;  // rows whose results are not finite
    static constexpr int kOffSeg = kOffAgain + 32 * 4;
    static constexpr int kOffBar = kOffSeg + kSegs * int(sizeof(Segment));
    static constexpr int kBars = 2 * kSlots + 2 * kSegs + 6;
    static constexpr int kBytes = kOffBar + kBars * 8 + 16;
    static constexpr int kAlloc = kBytes + 1024;     // the base is rounded up to 1024
    static_assert(kAlloc <= 115712, "two blocks per SM");
};

template <int DP, bool BF>
__global__ void __launch_bounds__(Shape<DP>::kThreads, 2)
    k_light(const sim_kv kv, const sim_kv_batch b, const KvAttend a, const __grid_constant__ KvMaps maps) {
    using Sh = Shape<DP>;
    constexpr int NS = Sh::kSlots, NK = kv_tile(1);
    extern __shared__ unsigned char raw[];
    unsigned char *const base = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
    const uint32_t sbase = smem_addr(base), bars = sbase + Sh::kOffBar;
    volatile int *const gave_up = reinterpret_cast<int *>(base + Sh::kOffBar + Sh::kBars * 8);
    uint32_t *const tmem_at = reinterpret_cast<uint32_t *>(base + Sh::kOffBar + Sh::kBars * 8 + 4);
    Segment *const segs = reinterpret_cast<Segment *>(base + Sh::kOffSeg);
    const auto full = [&](uint32_t slot) { return bars + 8 * slot; };
    const auto empty = [&](uint32_t slot) { return bars + 8 * (NS + slot); };
    const auto seg_full = [&](uint32_t x) { return bars + 8 * (2 * NS + x % kSegs); };
    const auto seg_empty = [&](uint32_t x) { return bars + 8 * (2 * NS + kSegs + x % kSegs); };
    constexpr int kRest = 2 * NS + 2 * kSegs;
    const uint32_t q_full = bars + 8 * kRest, s_full = q_full + 8, p_ready = q_full + 16, o_full = q_full + 24, drained = q_full + 32, joined = q_full + 40;
    const int tid = threadIdx.x, warp = __shfl_sync(FULL, tid >> 5, 0), lane = tid & 31;

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int s = 0; s < kSegs; ++s) {
            bar_init(seg_full(s), 1);
            bar_init(seg_empty(s), 5);
        }
        bar_init(q_full, 4);
        bar_init(s_full, 1);
        bar_init(p_ready, 4);
        bar_init(o_full, 1);
        bar_init(drained, 1);
        bar_init(joined, 4);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 128) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.keys) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.values) : "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_at)), "n"(Sh::kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(FULL, *tmem_at, 0);
    kv_wait_previous();

    const int G = b.q_heads / kv.n_kv_heads, D = kv.head_dim;
    // Segment number x, for the warps that are told of it, until each of them gives it back.
    const auto take = [&](uint32_t x) { return __all_sync(FULL, bar_wait(seg_full(x), (x / kSegs) & 1, gave_up)) != 0; };
    const auto give_back = [&](uint32_t x) {
        __syncwarp();
        if (lane == 0) bar_arrive(seg_empty(x));
    };
    // A slot of the ring and the parity of its current use.
    struct Ring {
        uint32_t slot = 0, parity = 0;
        __device__ void next() {
            if (++slot == NS) {
                slot = 0;
                parity ^= 1;
            }
        }
    };

    if (warp == 4) {
        // ---- the line of work, and loads: lane l brings page l of each tile
        const KvPlan plan = kv_plan(kv, b);
        Line line(plan, kv.n_kv_heads, 1, blockIdx.x, a.sms);
        const int P = kv.page_size, box = min(P, NK), per = NK / box;
        Ring ring;
        uint32_t used = 0;
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
            const auto page_of = [&](int j) {  // of this lane in tile j; past the keys: none, zeros
                const int key = sg.k0 + j * NK + lane * box;
                return lane < per && j < sg.n && key < sg.kv1 ? row[key / P] : -1;
            };
            int page = page_of(0);
            for (int j = 0; j < sg.n && ok; ++j) {
                const int next_page = page_of(j + 1), inside = (sg.k0 + j * NK + lane * box) % P;
                const int w = unsigned(page) < unsigned(kv.n_pages) ? page : kv.n_pages;
#pragma unroll
                for (int v = 0; v < 2; ++v) {  // keys, values
                    ok = __all_sync(FULL, bar_wait(empty(ring.slot), ring.parity ^ 1, gave_up));
                    if (!ok) break;
                    if (lane == 0) bar_expect(full(ring.slot), Sh::kTile);
                    __syncwarp();
                    if (lane < per) {
                        const uint32_t dst = sbase + ring.slot * Sh::kTile + lane * box * 128;
#pragma unroll
                        for (int half = 0; half < DP / 64; ++half)
                            tma_load(dst + half * Sh::kHalf, v ? &maps.values : &maps.keys, full(ring.slot), half * 64, inside, sg.h, w);
                    }
                    ring.next();
                    ++used;
                }
                page = next_page;
            }
        }
        if (!ok) {  // let what is on its way arrive
            for (uint32_t k = used > NS ? used - NS : 0; k < used; ++k)
                for (int n = 0; n < 1000000 && !bar_try(full(k % NS), (k / NS) & 1); ++n) {
                }
            if (lane == 0) atomicMin(kv.status, SIM_E_STATE);
        }
    } else if (warp == 5) {
        // ---- tensor products: the whole warp keeps the same (uniform) state, one lane issues
        const uint32_t type = BF ? 1u << 7 | 1u << 10 : 0u;
        const uint32_t idesc_s = 1u << 4 | type | (NK / 8) << 17 | (128 / 16) << 24;
        const uint32_t idesc_o = 1u << 4 | type | 1u << 16 | (DP / 8) << 17 | (128 / 16) << 24;
        const uint64_t op_k = operand(sbase, 16, 1024), op_v = operand(sbase, Sh::kHalf, 1024);
        Ring ring;
        uint32_t np = 0;
        bool ok = true;
        const auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(FULL, bar_wait(bar, parity, gave_up)) != 0; };
        const auto keys = [&] {  // S of the tile in the ring's slot
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk)
                    mma_ts(tmem, tmem + Sh::kColQ + kk * 8, op_k + ((ring.slot * Sh::kTile + (kk / 4) * Sh::kHalf + (kk % 4) * 32) >> 4), idesc_s, kk > 0);
                tc_commit(s_full);
                tc_commit(empty(ring.slot));
            }
            __syncwarp();
            ring.next();
        };
        for (uint32_t x = 0; (ok = take(x)); ++x) {
            const int n = __shfl_sync(FULL, segs[x % kSegs].n, 0);
            give_back(x);
            if (n == 0) break;
            ok = wait(q_full, x & 1) && wait(full(ring.slot), ring.parity);
            if (!ok) break;
            tc_fence_after();
            keys();
            for (int j = 0; j < n && ok; ++j, ++np) {
                ok = wait(full(ring.slot), ring.parity) && wait(p_ready, np & 1);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < NK / 16; ++kk)
                        mma_ts(tmem + Sh::kColO, tmem + kk * 8, op_v + ((ring.slot * Sh::kTile + kk * 2048) >> 4), idesc_o, j > 0 || kk > 0);
                    tc_commit(empty(ring.slot));
                    if (j + 1 == n) tc_commit(o_full);
                }
                __syncwarp();
                ring.next();
                if (j + 1 < n) {
                    ok = wait(full(ring.slot), ring.parity);
                    if (!ok) break;
                    keys();
                }
            }
            if (!ok) break;
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
        // ---- queries, softmax, results
        const int w = warp, lr = tid;
        const uint32_t t_s = tmem + (uint32_t(w * 32) << 16), t_q = t_s + Sh::kColQ, t_o = t_s + Sh::kColO;
        float *const stage = reinterpret_cast<float *>(base + Sh::kOffStage);
        float2 *const stat = reinterpret_cast<float2 *>(base + Sh::kOffStat);
        int *const again = reinterpret_cast<int *>(base + Sh::kOffAgain);
        const float c = a.scale_log2;
        uint32_t ns = 0, nj = 0;
        Ring ring;  // of the tile's keys
        bool ok = true;
        const auto join = [&] {  // the four warps, by a barrier whose wait ends even if some have given up
            __syncwarp();
            if (lane == 0) bar_arrive(joined);
            ok = __all_sync(FULL, bar_wait(joined, nj++ & 1, gave_up)) && ok;
        };
        // The query row in this thread's lane.
        const auto q_row = [&](const Segment &s) {
            const int y = s.row0 + min(lane, s.rows - 1), t = a.group.div(y);
            return static_cast<const uint16_t *>(a.q) + int64_t(s.q0 + t) * a.qt + int64_t(s.h * G + y - t * G) * a.qh;
        };
        const auto load_q = [&](const Segment &s) {
            const uint16_t *from = q_row(s);
            if (a.q_vec) {
#pragma unroll
                for (int half = 0; half < DP / 64; ++half) {
                    uint4 q[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[j] = half * 64 + j * 8 < D ? *reinterpret_cast<const uint4 *>(from + half * 64 + j * 8) : make_uint4(0, 0, 0, 0);
                    tm_st32(t_q + 32 * half, reinterpret_cast<const uint32_t *>(q));
                }
            } else {
#pragma unroll 1
                for (int d = 0; d < DP; d += 16) {
                    uint32_t q[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[j] = d + 2 * j < D ? from[d + 2 * j] | uint32_t(from[d + 2 * j + 1]) << 16 : 0;
                    tm_st8(t_q + d / 2, q);
                }
            }
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(q_full);
        };
        // Before segment 0 comes one without tiles, so that the code that takes up the next segment is there once.
        for (uint32_t x = ~0u; ok; ++x) {
            const Segment &sg = segs[x % kSegs], &next = segs[(x + 1) % kSegs];
            const bool real = x != ~0u;
            const int n = real ? sg.n : 0;
            if (real && n == 0) break;
            const int rows = sg.rows;
            // key position that it sees last; lanes past the rows see all: theirs are no reason to mask a tile
            const int last = lane < rows ? min(sg.kv1 - 1, sg.pos0 + int(a.group.div(sg.row0 + lane))) : sg.kv1 - 1;
            float m = -INFINITY, l = 0.f;
            if (!real) ok = take(0);
            int k0 = sg.k0;  // first key of the tile
            const int kv1 = sg.kv1;
            for (int j = 0; j < n; ++j, k0 += NK) {
                if (j == max(n - 2, 0)) {  // the next item's queries come to L1 meanwhile: two lines a row
                    ok = take(x + 1);
                    if (!ok) break;
                    if (next.n > 0 && lr < next.rows) {
                        const uint16_t *from = q_row(next);
                        uint16_t v;
                        asm volatile("ld.global.ca.u16 %0, [%1];" : "=h"(v) : "l"(from));
                        asm volatile("ld.global.ca.u16 %0, [%1];" : "=h"(v) : "l"(from + D - 1));
                    }
                }
                ok = __all_sync(FULL, bar_wait(s_full, ns & 1, gave_up));
                if (!ok) break;
                ++ns;
                tc_fence_after();
                softmax_tile<NK, 4, DP, BF>(t_s, t_o, w, last - k0 - w * (NK / 4), j == 0, c, m, l, [] {});
                ring.next();
                // values past the end of the keys, whatever they are, must not meet their zero probabilities
                const int valid = kv1 - k0;
                if (valid < NK) {
                    ok = __all_sync(FULL, bar_wait(full(ring.slot), ring.parity, gave_up));
                    if (lr >= 2 * valid) {  // two threads a row
                        unsigned char *v = base + ring.slot * Sh::kTile + (lr >> 1) * 128 + (lr & 1) * 64;
#pragma unroll
                        for (int z = 0; z < DP / 16; ++z) *reinterpret_cast<uint4 *>(v + (z / 4) * Sh::kHalf + (z % 4) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    smem_to_async();
                }
                ring.next();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_ready);
            }
            if (!ok) break;
            if (next.n > 0) load_q(next);  // every product with this item's queries has been read
            if (!real) continue;

            const Sink<BF> sink = {kv, a, sg, G, D, b.q_heads, sg.k0 + n * NK};
            // Join the four copies of each row: first what each is multiplied by.
            float2 *const st = stat + (x & 1) * 128;
            st[lr] = make_float2(m, l);
            join();
            float top = -INFINITY, total = 0.f;
#pragma unroll
            for (int p = 0; p < 4; ++p)
                if (st[32 * p + lane].y != 0.f) top = fmaxf(top, st[32 * p + lane].x);
#pragma unroll
            for (int p = 0; p < 4; ++p)
                if (st[32 * p + lane].y != 0.f) total += st[32 * p + lane].y * ex2((st[32 * p + lane].x - top) * c);
            const float f = l == 0.f ? 0.f : ex2((m - top) * c) / total;
            if (lr < rows) sink.lse(lr, top, total);
            if (lr < 32) again[lr] = 0;
            // As many columns at a time as the stage holds of all copies.  No wait is needed after the last ones: the stage is
            // used again only after the other warps have gone on to another item.
            int cols = DP, shift = DP == 128 ? 5 : 4;  // log2 of the columns / 4
            while (4 * rows * (cols + 4) > Sh::kJoinStage) {
                cols /= 2;
                --shift;
            }
            float *const to = stage + (w * rows + lane) * (cols + 4);
            ok = __all_sync(FULL, bar_wait(o_full, x & 1, gave_up)) && ok;
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int d0 = 0; d0 < D; d0 += cols) {
                if (d0 > 0) join();
#pragma unroll 1
                for (int d = 0; d < cols; d += 32) {
                    uint32_t o[32];
                    if (cols == 16) tm_ld16(t_o + d0, o);
                    else tm_ld32(t_o + d0 + d, o);
                    tc_wait_ld();
                    if (lane < rows) {
#pragma unroll
                        for (int y = 0; y < 32; y += 4)
                            if (y < 16 || cols > 16)
                                *reinterpret_cast<float4 *>(to + d + y) =
                                    l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)
                                             : make_float4(__uint_as_float(o[y]) * f, __uint_as_float(o[y + 1]) * f, __uint_as_float(o[y + 2]) * f, __uint_as_float(o[y + 3]) * f);
                    }
                }
                join();
                if (!ok) break;
#pragma unroll 1
                for (int e = lr; e < rows << shift; e += 128) {
                    const int y = e >> shift, d = 4 * (e & ((1 << shift) - 1));
                    if (d0 + d >= D) continue;
                    float4 v[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) v[p] = *reinterpret_cast<const float4 *>(stage + (p * rows + y) * (cols + 4) + d);
                    const float4 t = make_float4((v[0].x + v[1].x) + (v[2].x + v[3].x), (v[0].y + v[1].y) + (v[2].y + v[3].y),
                                                 (v[0].z + v[1].z) + (v[2].z + v[3].z), (v[0].w + v[1].w) + (v[2].w + v[3].w));
                    if (sg.direct) *reinterpret_cast<uint2 *>(sink.out_row(y) + d0 + d) = make_uint2(pack<BF>(t.x, t.y), pack<BF>(t.z, t.w));
                    else *reinterpret_cast<float4 *>(a.part + (sg.row + y) * D + d0 + d) = t;
                    if (t.x * 0.f + t.y * 0.f + t.z * 0.f + t.w * 0.f != 0.f) again[y] = 1;
                }
            }
            if (!ok) break;
            if (sink.blind(0)) {  // see Sink::again
                join();
                if (!ok) break;
                for (int y = w; y < rows; y += 4)
                    if (again[y] && sink.blind(y)) sink.again(y);
            }
            tc_fence_before();
            give_back(x);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Sh::kTmem));
    }
}

template <int DP, bool BF>
cudaError_t launch(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, const KvMaps &maps, cudaStream_t st) {
    static thread_local int ready = -1;  // the device on which the kernel has its shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev != ready) {
        e = cudaFuncSetAttribute((const void *)k_light<DP, BF>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP>::kAlloc);
        if (e == cudaSuccess) ready = dev;
    }
    return e == cudaSuccess ? launch_chained(k_light<DP, BF>, kv_blocks(a.sms, 1), Shape<DP>::kThreads, Shape<DP>::kAlloc, st, kv, b, a, maps) : e;
}

}  // namespace

cudaError_t launch_kv_light(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, const KvMaps &maps, cudaStream_t st) {
    if (kv.dtype == SIM_KV_BF16) return kv.head_dim > 64 ? launch<128, true>(kv, b, a, maps, st) : launch<64, true>(kv, b, a, maps, st);
    return kv.head_dim > 64 ? launch<128, false>(kv, b, a, maps, st) : launch<64, false>(kv, b, a, maps, st);
}

}  // namespace simgb
