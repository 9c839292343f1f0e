// Attention of light items (up to 32 query rows; see sim_kv_attend.cu): single tokens of one sequence and the
// few rows of small groups, bound by the bytes of the keys and values.
//
// Keys take the 128 rows of the tensor products, queries their columns, so that few queries cost little.  Per tile of
// 128 keys: S' = K Q' (128 x N x D, N = 16 or 32), P' = exp2(c (S' - m)), a thread for each key, O' += V' P' (D x N x 128, V as
// it lies, its M dimension contiguous).  P goes to shared memory, over the tile's first keys, which are no longer needed.
// A row's keys lie in all of the block's threads: its sum is joined at the end of the item, its maximum in the item's first
// tile and then only where a key exceeds it by more than kGrow, which the four warps tell each other in every tile.  Eight
// rows are in registers at a time, whatever their number; each thread's own sums wait in TMEM.
// Two blocks per SM, so that one loads while the other is between two items, with 96 KB of keys and values in flight each.
// Rows of P are rounded as in sim_kv_heavy.cu.
//
// 384 sequences of up to 2600 keys, 8 query heads on each of 8 kv heads, D = 128: 316 us for 2.10 GB, 6.64 TB/s; one sequence
// of 131071 keys 80 us for 0.54 GB, 6.7 TB/s: what a copy reaches.  With queries on the rows (each four times, for four
// quarters of the keys) these took 330 and 85 us.  D <= 64 has half the columns: the first with D = 64 takes 197 us with the plan, 223 us as D = 128.
#include "sim_kv_attend.cuh"

namespace simgb {

namespace {

template <int DP>
struct Shape {
    static constexpr int kThreads = 192;              // four softmax warps, one loads, one issues
    static constexpr int kHalves = DP / 64;
    static constexpr int kSlot = 16384;               // 64 columns of 128 keys or values
    static constexpr int kSlots = 6;
    static constexpr int kRowsHalf = kLightRows * 128;  // 64 columns of the queries, or 64 keys of P
    static constexpr int kTmem = 128, kColO = 32, kColL = 64;  // S below; L: each thread's sums
    static constexpr int kOffQ = kSlots * kSlot;
    static constexpr int kOffRed = kOffQ + kHalves * kRowsHalf;  // [2][row][warp]
    static constexpr int kOffVote = kOffRed + 2 * kLightRows * 16;
    static constexpr int kOffBad = kOffVote + 2 * 16;  // keys with values that are not finite, in tiles that not all rows see whole
    static constexpr int kOffSeg = kOffBad + kBlindTiles * 16;
    static constexpr int kOffBar = kOffSeg + kSegs * int(sizeof(Segment));
    static constexpr int kBars = 2 * kSlots + 2 * kSegs + 6;
    static constexpr int kBytes = kOffBar + kBars * 8 + 16;
    static constexpr int kAlloc = kBytes + 1024;      // the base is rounded up to 1024
    static_assert(kAlloc <= 115712, "two blocks per SM");
    static_assert(kSlots % (2 * kHalves) % kHalves == 0, "the halves of a tile lie side by side");
};

// Eight rows' maxima or sums over the warp's lanes: row lane / 4's is returned.
template <bool SUM>
__device__ __forceinline__ float over_lanes(const float *x) {
    const int lane = threadIdx.x & 31;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
#pragma unroll
    for (int d = 16, n = 4; d >= 1; d /= 2, n /= 2) {
        if (n >= 1) {
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const bool up = lane & d;
                const float mine = up ? v[i + n] : v[i], other = __shfl_xor_sync(FULL, up ? v[i] : v[i + n], d);
                v[i] = SUM ? mine + other : fmaxf(mine, other);
            }
        } else {
            const float other = __shfl_xor_sync(FULL, v[0], d);
            v[0] = SUM ? v[0] + other : fmaxf(v[0], other);
        }
    }
    return v[0];
}

template <int DP, bool BF>
__global__ void __launch_bounds__(Shape<DP>::kThreads, 2)
    k_light(const sim_kv kv, const sim_kv_batch b, const KvAttend a, const __grid_constant__ KvMaps maps) {
    using Sh = Shape<DP>;
    constexpr int NS = Sh::kSlots, HF = Sh::kHalves, NK = kTileKeys;
    extern __shared__ unsigned char raw[];
    unsigned char *const base = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
    const uint32_t sbase = smem_addr(base), bars = sbase + Sh::kOffBar;
    volatile int *const gave_up = reinterpret_cast<int *>(base + Sh::kOffBar + Sh::kBars * 8);
    uint32_t *const tmem_at = reinterpret_cast<uint32_t *>(base + Sh::kOffBar + Sh::kBars * 8 + 4);
    Segment *const segs = reinterpret_cast<Segment *>(base + Sh::kOffSeg);
    const auto full = [&](uint32_t x) { return bars + 8 * (x % NS); };
    const auto empty = [&](uint32_t x) { return bars + 8 * (NS + x % NS); };
    const auto slot_at = [&](uint32_t x) { return sbase + (x % NS) * Sh::kSlot; };
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
        bar_init(o_full, 2);
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
    if (warp == 4) {
        // ---- the line of work, and loads: lane l brings page l of each tile
        const KvPlan plan = kv_plan(kv, b);
        Line line(plan, kv.n_kv_heads, 1, blockIdx.x, a.sms);
        const int P = kv.page_size, per = NK / P;
        uint32_t at = 0;  // slots loaded: for each tile the halves of the keys, of the values
        bool ok = true;
        const auto tell = [&](uint32_t x, const Segment &sg) {
            ok = __all_sync(FULL, bar_wait(seg_empty(x), (x / kSegs + 1) & 1, gave_up));
            if (ok && lane == 0) {
                segs[x % kSegs] = sg;
                bar_arrive(seg_full(x));
            }
        };
        Segment sg, ahead;
        line.next(sg);
        tell(0, sg);
        for (uint32_t x = 0; ok && sg.n > 0; ++x, sg = ahead) {
            // The next segment is told of before this one is loaded: the softmax asks for it while this one's last tiles wait
            // for slots that its own work has to free.
            line.next(ahead);
            tell(x + 1, ahead);
            const int32_t *row = kv.table + int64_t(sg.seq) * kv.max_pages;
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
                for (int y = 0; y < 2 * HF; ++y, ++at) {
                    ok = __all_sync(FULL, bar_wait(empty(at), (at / NS + 1) & 1, gave_up));
                    if (!ok) break;
                    if (lane == 0) bar_expect(full(at), Sh::kSlot);
                    __syncwarp();
                    if (lane < per) tma_load(slot_at(at) + lane * P * 128, y < HF ? &maps.keys : &maps.values, full(at), y % HF * 64, 0, sg.h, w);
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
    } else if (warp == 5) {
        // ---- tensor products: the whole warp keeps the same (uniform) state, one lane issues
        const uint32_t type = BF ? 1u << 7 | 1u << 10 : 0u;
        const uint32_t op_q = sbase + Sh::kOffQ;
        uint32_t at = 0, np = 0;
        bool ok = true;
        const auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(FULL, bar_wait(bar, parity, gave_up)) != 0; };
        const auto wait_full = [&](uint32_t x) {
            bool all = true;
#pragma unroll
            for (int y = 0; y < HF; ++y) all = all && wait(full(x + y), ((x + y) / NS) & 1);
            return all;
        };
        for (uint32_t x = 0; (ok = take(x)); ++x) {
            const int n = __shfl_sync(FULL, segs[x % kSegs].n, 0), cols = __shfl_sync(FULL, segs[x % kSegs].rows, 0) > 16 ? 32 : 16;
            give_back(x);
            if (n == 0) break;
            const uint32_t idesc_s = 1u << 4 | type | uint32_t(cols / 8) << 17 | (128 / 16) << 24, idesc_o = idesc_s | 1u << 15;
            ok = wait(q_full, x & 1);
            for (int j = 0; j < n && ok; ++j, ++np, at += 2 * HF) {
                ok = wait_full(at);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk)
                        mma_ss(tmem, operand(slot_at(at + kk / 4) + kk % 4 * 32, 16, 1024), operand(op_q + (kk / 4) * Sh::kRowsHalf + kk % 4 * 32, 16, 1024), idesc_s, kk > 0);
                    tc_commit(s_full);
#pragma unroll
                    for (int y = 1; y < HF; ++y) tc_commit(empty(at + y));  // P takes the first half's place
                }
                __syncwarp();
                ok = wait_full(at + HF) && wait(p_ready, np & 1);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    // D <= 64: rows 64 .. 127 of the product are made of other values (8 keys on) and not used
#pragma unroll
                    for (int kk = 0; kk < NK / 16; ++kk)
                        mma_ss(tmem + Sh::kColO, operand(slot_at(at + HF) + kk * 2048, HF > 1 ? Sh::kSlot : 1024, 1024),
                               operand(slot_at(at) + (kk / 4) * Sh::kRowsHalf + kk % 4 * 32, 16, 1024), idesc_o, j > 0 || kk > 0);
                    tc_commit(empty(at));
#pragma unroll
                    for (int y = HF; y < 2 * HF; ++y) tc_commit(empty(at + y));
                    if (j + 1 == n) {
                        tc_commit(o_full);
                        bar_arrive(o_full);  // what the warps have told each other in shared memory is there as well
                    }
                }
                __syncwarp();
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
        const int w = warp, lr = tid;  // the key within a tile, the column of the result
        const uint32_t t_s = tmem + (uint32_t(w * 32) << 16), t_o = t_s + Sh::kColO;
        float *const red = reinterpret_cast<float *>(base + Sh::kOffRed);
        int *const vote = reinterpret_cast<int *>(base + Sh::kOffVote);
        uint32_t *const bad = reinterpret_cast<uint32_t *>(base + Sh::kOffBad);
        const float c = a.scale_log2;
        uint32_t ns = 0, nj = 0, nr = 0, nv = 0, at = 0;
        bool ok = true;
        const auto join = [&] {  // the four warps, by a barrier whose wait ends even if some have given up
            __syncwarp();
            if (lane == 0) bar_arrive(joined);
            ok = __all_sync(FULL, bar_wait(joined, nj++ & 1, gave_up)) && ok;
        };
        // Queries: 16 bytes of a row at a time, the next item's fetched before they can be put in place.
        constexpr int kVec = DP / 8, kFetch = kLightRows * kVec / 128;
        uint4 query[kFetch];
        const auto query_at = [&](const Segment &s, int i) {  // this thread's i-th 16 bytes, NULL if there are none
            const int r = (lr + 128 * i) / kVec, d = (lr + 128 * i) % kVec * 8, y = s.row0 + r, t = a.group.div(y);
            return r < s.rows && d < D ? static_cast<const uint16_t *>(a.q) + int64_t(s.q0 + t) * a.qt + int64_t(s.h * G + y - t * G) * a.qh + d : nullptr;
        };
        const auto fetch = [&](const Segment &s) {
#pragma unroll
            for (int i = 0; i < kFetch; ++i) {
                const uint16_t *from = a.q_vec ? query_at(s, i) : nullptr;
                query[i] = from ? *reinterpret_cast<const uint4 *>(from) : make_uint4(0, 0, 0, 0);  // columns past the head's: zeros
            }
        };
        const auto place = [&](const Segment &s) {
            const auto put = [&](int i, uint4 v) {
                const int r = (lr + 128 * i) / kVec, e = (lr + 128 * i) % kVec;
                if (r < s.rows) *reinterpret_cast<uint4 *>(base + Sh::kOffQ + (e / 8) * Sh::kRowsHalf + r * 128 + ((e % 8 ^ (r & 7)) << 4)) = v;
            };
            if (a.q_vec) {
#pragma unroll
                for (int i = 0; i < kFetch; ++i) put(i, query[i]);
            } else {
#pragma unroll 1
                for (int i = 0; i < kFetch; ++i) {
                    const uint16_t *from = query_at(s, i);
                    put(i, from ? make_uint4(from[0] | uint32_t(from[1]) << 16, from[2] | uint32_t(from[3]) << 16, from[4] | uint32_t(from[5]) << 16,
                                             from[6] | uint32_t(from[7]) << 16)
                                : make_uint4(0, 0, 0, 0));
                }
            }
            smem_to_async();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(q_full);
        };
        ok = take(0);
        if (ok && segs[0].n > 0) {
            fetch(segs[0]);
            place(segs[0]);
        }
        for (uint32_t x = 0; ok; ++x) {
            const Segment &sg = segs[x % kSegs], &next = segs[(x + 1) % kSegs];
            const int n = sg.n, rows = sg.rows, kv1 = sg.kv1;
            if (n == 0) break;
            // The first key that row `lane` does not see; that row 0 does not.
            const int blind = min(kv1, sg.pos0 + int(a.group.div(sg.row0 + lane)) + 1), all = __shfl_sync(FULL, blind, 0);
            int k0 = sg.k0;  // first key of the tile
            // Eight rows' scores of this thread's key, -infinity where they do not see it.
            const auto scores = [&](int r0, float *s) {
                uint32_t u[8];
                tm_ld8(t_s + r0, u);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = __uint_as_float(u[i]);
                if (k0 + NK > all) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] = k0 + lr >= __shfl_sync(FULL, blind, r0 + i) ? -INFINITY : s[i];
                }
            };
            // A row's maximum or sum over all of the block's keys, for the lane of that number.  Between two uses of one half
            // of `red` lies a third one.
            const auto joined_rows = [&](auto sum) {
                constexpr bool SUM = decltype(sum)::value;
                float *const to = red + (++nr & 1) * kLightRows * 4;
#pragma unroll 1
                for (int r0 = 0; r0 < rows; r0 += 8) {
                    float s[8];
                    if constexpr (SUM) {
                        uint32_t u[8];
                        tm_ld8(t_s + Sh::kColL + r0, u);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 8; ++i) s[i] = __uint_as_float(u[i]);
                    } else {
                        scores(r0, s);
                    }
                    const float v = over_lanes<SUM>(s);
                    if (lane % 4 == 0) to[(r0 + lane / 4) * 4 + w] = v;
                }
                join();
                const float4 v = *reinterpret_cast<const float4 *>(to + lane * 4);
                return SUM ? (v.x + v.y) + (v.z + v.w) : fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w));
            };
            const Sink<BF> sink = {kv, a, sg, G, D, b.q_heads};
            const int blind_from = sink.blind_from();
            float m = -INFINITY;  // of row `lane`: log2, times c
#pragma unroll 1
            for (int j = 0; j < n; ++j, k0 += NK, at += 2 * HF) {
                if (j == max(n - 2, 0)) {
                    ok = take(x + 1);
                    if (!ok) break;
                    if (next.n > 0) fetch(next);
                }
                ok = __all_sync(FULL, bar_wait(s_full, ns++ & 1, gave_up));
                if (!ok) break;
                tc_fence_after();
                bool grows = j == 0;
                if (j > 0) {
#pragma unroll 1
                    for (int r0 = 0; r0 < rows; r0 += 8) {
                        float s[8];
                        scores(r0, s);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float over = fmaf(s[i], c, -__shfl_sync(FULL, m, r0 + i));
                            grows |= r0 + i < rows && over > kGrow;
                        }
                    }
                    grows = __any_sync(FULL, grows);
                    int *const to = vote + (nv++ & 1) * 4;
                    if (lane == 0) to[w] = grows;
                    join();
                    if (!ok) break;
                    const int4 v = *reinterpret_cast<const int4 *>(to);
                    grows = v.x | v.y | v.z | v.w;
                }
                if (grows) {
                    const float top = joined_rows(std::false_type()) * c;
                    if (!ok) break;
                    // each row for itself: what it becomes does not hang on the rows beside it
                    const bool up = j == 0 || top - m > kGrow;
                    const float f = up ? ex2(m - top) : 1.f;
                    if (up) m = top;
#pragma unroll 1
                    for (int r0 = 0; r0 < rows && j > 0; r0 += 8) {  // O: the product before has ended, this tile's first came after it
                        uint32_t o[8], l[8];
                        tm_ld8(t_o + r0, o);
                        tm_ld8(t_s + Sh::kColL + r0, l);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float fi = __shfl_sync(FULL, f, r0 + i);
                            o[i] = __float_as_uint(__uint_as_float(o[i]) * fi);
                            l[i] = __float_as_uint(__uint_as_float(l[i]) * fi);
                        }
                        tm_st8(t_o + r0, o);
                        tm_st8(t_s + Sh::kColL + r0, l);
                        tc_wait_st();
                    }
                }
                unsigned char *const p = base + (at % NS) * Sh::kSlot + lr / 64 * Sh::kRowsHalf + lr % 8 * 2;
                const float off = m == -INFINITY ? 0.f : kv_lift(BF) - m;
#pragma unroll 1
                for (int r0 = 0; r0 < rows; r0 += 8) {
                    float s[8];
                    uint32_t l[8] = {};
                    if (j > 0) tm_ld8(t_s + Sh::kColL + r0, l);
                    scores(r0, s);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        s[i] = ex2(fmaf(s[i], c, __shfl_sync(FULL, off, r0 + i)));
                        l[i] = __float_as_uint(__uint_as_float(l[i]) + s[i]);
                    }
                    tm_st8(t_s + Sh::kColL + r0, l);
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const uint32_t both = pack<BF>(s[i], s[i + 1]);
                        *reinterpret_cast<uint16_t *>(p + (r0 + i) * 128 + ((lr % 64 / 8 ^ i) << 4)) = uint16_t(both);
                        *reinterpret_cast<uint16_t *>(p + (r0 + i + 1) * 128 + ((lr % 64 / 8 ^ (i + 1)) << 4)) = uint16_t(both >> 16);
                    }
                }
                // values past the end of the keys, whatever they are, must not meet their zero probabilities, nor those that are
                // not finite the rows that do not see them
                if (kv1 - k0 < NK || j >= blind_from) {
#pragma unroll
                    for (int y = HF; y < 2 * HF; ++y) ok = __all_sync(FULL, bar_wait(full(at + y), ((at + y) / NS) & 1, gave_up)) && ok;
                    if (!ok) break;
                    unsigned char *const v = base + ((at + HF) % NS) * Sh::kSlot + lr * 128;
                    bool found = false;
                    if (lr >= kv1 - k0) {
#pragma unroll
                        for (int z = 0; z < DP / 8; ++z) *reinterpret_cast<uint4 *>(v + z / 8 * Sh::kSlot + z % 8 * 16) = make_uint4(0, 0, 0, 0);
                    } else if (j >= blind_from) {
                        found = clean_row<DP, BF>(v, Sh::kSlot);
                    }
                    if (j >= blind_from) {
                        const unsigned keys = __ballot_sync(FULL, found);
                        if (lane == 0) bad[(j - blind_from) * 4 + w] = keys;
                    }
                }
                tc_wait_st();
                smem_to_async();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_ready);
            }
            if (!ok) break;
            if (next.n > 0) place(next);  // every product with this item's queries has ended

            const float before = lane < rows ? sink.before(lane) : -INFINITY;  // written anew only after the next join
            const typename Sink<BF>::Joint joint = sink.joint(m - kv_lift(BF), joined_rows(std::true_type()), before);
            ok = __all_sync(FULL, bar_wait(o_full, x & 1, gave_up)) && ok;
            if (!ok) break;
            tc_fence_after();
            if (lr < rows) sink.lse(lr, joint.e);
            int h = sg.row0 - int(a.group.div(sg.row0)) * G;  // head of the row in its group
            uint16_t *out = sink.out_row(0) + lr;
            float *part = a.part + sg.row * D + lr;
#pragma unroll 1
            for (int r0 = 0; r0 < rows; r0 += 8) {
                uint32_t o[8];
                tm_ld8(t_o + r0, o);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float f = __shfl_sync(FULL, joint.mine, r0 + i), fb = __shfl_sync(FULL, joint.before, r0 + i);
                    float v = f == 0.f ? 0.f : __uint_as_float(o[i]) * f;
                    if (r0 + i < rows && lr < D) {
                        if (fb != 0.f) v = fmaf(*part, fb, v);
                        if (sg.direct) *out = uint16_t(pack<BF>(v, v));
                        else *part = v;
                    }
                    part += D;
                    out += a.oh;
                    if (++h == G) {
                        h = 0;
                        out += a.ot - G * a.oh;
                    }
                }
            }
            uint32_t some = 0;
#pragma unroll 1
            for (int z = 0; z < 4 * (n - blind_from); ++z) some |= bad[z];
            if (some) {
                join();  // after the results
                if (!ok) break;
                for (int y = w; y < rows; y += 4) sink.spoil(y, bad);
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
