// Attention of light items (up to 8 or 16 query rows, kv_light_rows; see sim_kv_attend.cu) over a 4-bit cache: single tokens of one sequence
// and the few rows of small groups.
//
// Keys and values become 16-bit floats in registers, in the very places that the matrix instructions take their first operand
// from: the strips are laid out for that (include/sim_kv.h), so that a byte goes from HBM through shared memory into a register and no
// further.  (The tensor unit of sim_kv_heavy.cu takes its operands from shared memory: unpacked values would pass it three times, at 2
// bytes each, which at 128 bytes a cycle is all that it can give at HBM's rate.)  Per warp and strip of 16 keys: S' = K Q' (16 keys x 8 query
// rows at a time, D / 16 products), P' = exp2(c S' + off), whose 8 x 8 parts are turned over between the lanes, and O' += V' P' (D x 8, a
// product for each 16 columns).  Each warp keeps its own running maximum (as off), sum and O; the warps' shares are joined at the
// end of the segment.  P is rounded to the cache's type, its sum is not.
//
// 384 sequences of up to 2600 keys, 8 query heads on each of 8 kv heads, D = 128, bfloat16: 142 us for 0.62 GB, 4.4 TB/s (the 16-bit cache: 316
// us for 2.1 GB); one sequence of 131071 keys, float16: 38 us for 0.17 GB.  Unpacking bounds it: a strip's keys and values take a warp some 400
// instructions, of which 64 fused multiply-adds, 64 additions, 64 selections and 48 shifts (16 in float16) are on pipes that take two a
// cycle, and a mixture of these was measured at 2.9 to 3.05 a cycle; without loads the kernel takes 138 us, without arithmetic 107.  So it
// does not matter whether a warp takes one strip at a time or two (157.6 and 157.7 us, plan and join included) or whether the
// queries' exponents are computed once or twice.  When blocks were chosen (that call took 161 us then): three an SM 161, four with half
// tiles 166, two of eight warps 189 us.
#include <algorithm>
#include <cfloat>

#include "sim_kv_4bit.cuh"
#include "sim_kv_attend.cuh"

namespace simgb {

namespace {

constexpr int kStrips = kTileKeys / kStrip;  // of a tile

// DG groups of 32 columns, NT times 8 query rows (kv_light_rows), W warps that compute and one that loads.
template <int DG, int NT, int W>
struct Shape {
    static constexpr int kThreads = 32 * (W + 1);
    static constexpr int kRows = 8 * NT;
    static constexpr int kBytesStrip = 320 * DG;
    static constexpr int kStage = 2 * kStrips * kBytesStrip;  // a tile's keys, then its values
    static constexpr int kPitch = 32 * DG + 4;                // floats between rows of the warps' O
    static constexpr int kPerSm = NT == 1 ? 3 : 2;            // blocks, as in kv_per_sm
    static constexpr int kRoom = 233472 / kPerSm - 1024;
    // Queries and sums twice, so that one barrier for each part of a segment is enough.
    static constexpr int kSizeQ = NT * DG * 512, kSizeO = W * 8 * kPitch * 4, kSizeM = W * kRows * 8;
    static constexpr int kOffQ = 0;                           // queries: [NT][DG][lane] 16 bytes
    static constexpr int kOffO = kOffQ + 2 * kSizeQ;          // [W][8][kPitch]
    static constexpr int kOffM = kOffO + kSizeO;              // [W][kRows] off and sum
    static constexpr int kOffSeg = kOffM + 2 * kSizeM;
    static constexpr int kFixed = kOffSeg + kSegs * int(sizeof(Segment)) + 256;
    static constexpr int kStages = (kRoom - kFixed) / kStage < 8 ? (kRoom - kFixed) / kStage : 8;
    static constexpr int kOffRing = (kOffSeg + kSegs * int(sizeof(Segment)) + 127) / 128 * 128;
    static constexpr int kOffBar = kOffRing + kStages * kStage;
    static constexpr int kBars = 2 * kStages + 2 * kSegs + 2;
    static constexpr int kOffGone = kOffBar + kBars * 8;      // per stage: strips on pages that the pool does not have
    static constexpr int kBytes = kOffGone + kStages * 4 + 16;
    static_assert(kStages >= 2 && kBytes <= kRoom, "shared memory");
};

// 16 x 8 += 16 x 16 times 16 x 8.
template <bool BF>
__device__ __forceinline__ void product(float *d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The 8 x 8 matrix of which a lane has two values of row lane / 4, turned over.
__device__ __forceinline__ uint32_t turned(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <int DG, int NT, int W, bool BF>
__global__ void __launch_bounds__(Shape<DG, NT, W>::kThreads, Shape<DG, NT, W>::kPerSm)
    k_light_4bit(const sim_kv kv, const sim_kv_batch b, const KvAttend a) {
    using Sh = Shape<DG, NT, W>;
    constexpr int NS = Sh::kStages, R = Sh::kRows, KS = Sh::kBytesStrip;
    extern __shared__ __align__(128) unsigned char base[];
    const uint32_t sbase = smem_addr(base), bars = sbase + Sh::kOffBar;
    volatile int *const gave_up = reinterpret_cast<int *>(base + Sh::kOffGone + NS * 4);
    uint32_t *const gone = reinterpret_cast<uint32_t *>(base + Sh::kOffGone);
    Segment *const segs = reinterpret_cast<Segment *>(base + Sh::kOffSeg);
    const auto full = [&](uint32_t slot) { return bars + 8 * slot; };
    const auto empty = [&](uint32_t slot) { return bars + 8 * (NS + slot); };
    uint32_t slot = 0, turn = 0;  // of the ring
    const auto next_slot = [&] {
        slot = slot + 1 == NS ? 0 : slot + 1;
        turn ^= slot == 0;
    };
    const auto seg_full = [&](uint32_t x) { return bars + 8 * (2 * NS + x % kSegs); };
    const auto seg_empty = [&](uint32_t x) { return bars + 8 * (2 * NS + kSegs + x % kSegs); };
    const uint32_t joined = bars + 8 * (2 * NS + 2 * kSegs), cleared = joined + 8;
    const int tid = threadIdx.x, warp = __shfl_sync(FULL, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < NS; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), W);
        }
        for (int s = 0; s < kSegs; ++s) {
            bar_init(seg_full(s), 1);
            bar_init(seg_empty(s), W);
        }
        bar_init(joined, W);
        bar_init(cleared, W);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    kv_wait_previous();
    const int G = b.q_heads / kv.n_kv_heads, D = kv.head_dim;

    if (warp == W) {
        // ---- the line of work, and loads: lane l brings the keys of strip l, lane kStrips + l its values, those of a page's first
        // strip the others' of that page with them
        const KvPlan plan = kv_plan(kv, b);
        Line line(plan, kv.n_kv_heads, 1, blockIdx.x, a.sms);
        const int P = kv.page_size, strip = lane % kStrips, per = min(kStrips, P / kStrip);  // per: strips of a tile on one page
        const int64_t head_bytes = kv_head_bytes(kv), page_bytes = kv_page_bytes(kv);
        const unsigned char *const layer = static_cast<const unsigned char *>(kv.pool) + int64_t(a.layer) * 2 * kv.n_kv_heads * head_bytes;
        uint32_t x = 0;  // segments told of
        bool ok = true;
        const auto tell = [&](const Segment &sg) {
            ok = __all_sync(FULL, bar_wait(seg_empty(x), (x / kSegs + 1) & 1, gave_up));
            if (ok && lane == 0) {
                segs[x % kSegs] = sg;
                bar_arrive(seg_full(x));
            }
            ++x;
        };
        Segment sg, ahead;
        const auto page_of = [&](const Segment &s, int j) {  // of this lane's strip in tile j, -1 past the keys
            const int key = s.k0 + j * kTileKeys + strip * kStrip;
            return j < s.n && key < s.kv1 ? kv.table[int64_t(s.seq) * kv.max_pages + key / P] : -1;
        };
        line.next(sg);
        tell(sg);
        int page = page_of(sg, 0);
        while (ok && sg.n > 0) {
            // The next segment is told of, and its first pages are on their way, before this one is loaded.
            line.next(ahead);
            tell(ahead);
            for (int j = 0; j < sg.n && ok; ++j, next_slot()) {
                const int next_page = j + 1 < sg.n ? page_of(sg, j + 1) : page_of(ahead, 0), key = sg.k0 + j * kTileKeys + strip * kStrip;
                const bool in = key < sg.kv1, there = in && unsigned(page) < unsigned(kv.n_pages);
                ok = __all_sync(FULL, bar_wait(empty(slot), turn ^ 1, gave_up));
                if (!ok) break;
                const unsigned none = __ballot_sync(FULL, lane < kStrips && in && !there), some = __ballot_sync(FULL, lane < 2 * kStrips && there);
                if (lane == 0) {
                    gone[slot] = none;
                    bar_expect(full(slot), __popc(some) * KS);
                }
                __syncwarp();
                if (lane < 2 * kStrips && there && strip % per == 0)
                    bulk_load(sbase + Sh::kOffRing + slot * Sh::kStage + lane * KS,
                              layer + page * page_bytes + ((lane / kStrips) * kv.n_kv_heads + sg.h) * head_bytes + key % P / kStrip * KS,
                              KS * min(per, (sg.kv1 - key + kStrip - 1) / kStrip), full(slot));
                page = next_page;
            }
            sg = ahead;
        }
        if (!ok) {  // let what is on its way arrive
            for (int k = 0; k < NS; ++k, next_slot())  // (a slot that was never asked for is in its first turn, as is this wait)
                for (int n = 0; n < 1000000 && !bar_try(full(slot), turn ^ 1); ++n) {
                }
            if (lane == 0) atomicMin(kv.status, SIM_E_STATE);
        }
        return;
    }

    // ---- products, softmax, results: lane 4 g + t
    const int g = lane >> 2, t = lane & 3;
    const float c = a.scale_log2;
    uint32_t nj = 0, no = 0;
    bool ok = true;
    const auto join = [&] {  // the warps, by a barrier whose wait ends even if some have given up
        __syncwarp();
        if (lane == 0) bar_arrive(joined);
        ok = __all_sync(FULL, bar_wait(joined, nj++ & 1, gave_up)) && ok;
    };
    const auto take = [&](uint32_t x) { return __all_sync(FULL, bar_wait(seg_full(x), (x / kSegs) & 1, gave_up)) != 0; };
    // Queries, 8 columns of a row at a time: the second operand of two products; rows and columns that are not there are zeros.
    constexpr int kFetch = (NT * DG + W - 1) / W;
    uint4 query[kFetch];
    const auto fetch = [&](const Segment &s) {
#pragma unroll
        for (int e = 0; e < kFetch; ++e) {
            const int i = warp + W * e, j = i % DG, y = i / DG * 8 + g, d = 32 * j + 8 * t;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (y < s.rows && d < D) {
                const int z = s.row0 + y, tok = a.group.div(z);
                const uint16_t *from = static_cast<const uint16_t *>(a.q) + int64_t(s.q0 + tok) * a.qt + int64_t(s.h * G + z - tok * G) * a.qh + d;
                if (a.q_vec) v = *reinterpret_cast<const uint4 *>(from);
                else v = make_uint4(from[0] | uint32_t(from[1]) << 16, from[2] | uint32_t(from[3]) << 16, from[4] | uint32_t(from[5]) << 16,
                                    from[6] | uint32_t(from[7]) << 16);
            }
            query[e] = v;
        }
    };
    const auto queries = [&](uint32_t x) { return reinterpret_cast<uint4 *>(base + Sh::kOffQ + (x & 1) * Sh::kSizeQ); };
    const auto place = [&](uint32_t x) {
#pragma unroll
        for (int e = 0; e < kFetch; ++e)
            if (warp + W * e < NT * DG) queries(x)[(warp + W * e) * 32 + lane] = query[e];
    };
    ok = take(0);
    if (ok && segs[0].n > 0) {
        fetch(segs[0]);
        place(0);
        join();
    }
    for (uint32_t x = 0; ok; ++x) {
        const Segment &sg = segs[x % kSegs], &next = segs[(x + 1) % kSegs];
        const int n = sg.n, rows = sg.rows, kv1 = sg.kv1, first = sg.k0 + warp * (kStrips / W) * kStrip;  // this warp's first key
        if (n == 0) break;
        const Sink<BF, true> sink = {kv, a, sg, G, D, b.q_heads};
        const uint4 *const qs = queries(x);
        uint4 q1[NT == 1 ? DG : 1];  // 8 rows: in registers
        if constexpr (NT == 1)
#pragma unroll
            for (int j = 0; j < DG; ++j) q1[j] = qs[j * 32 + lane];
        const int all_see = sink.seen(0);  // keys that every row sees: rows are in the order of their tokens
        // off: what is added to a score, so that its power of two is its weight: 2^off is above one over the highest one's
        float o[NT][2 * DG][4], off[NT][2], sum[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
#pragma unroll
            for (int z = 0; z < 2 * DG; ++z) o[i][z][0] = o[i][z][1] = o[i][z][2] = o[i][z][3] = 0.f;
            off[i][0] = off[i][1] = FLT_MAX;
            sum[i][0] = sum[i][1] = 0.f;
        }
#pragma unroll 1
        for (int tile = 0; tile < n; ++tile, next_slot()) {
            if (tile == n - 1) {  // the next segment's queries are on their way while this one ends
                ok = take(x + 1);
                if (!ok) break;
                if (next.n > 0) fetch(next);
            }
            ok = __all_sync(FULL, bar_wait(full(slot), turn, gave_up));
            if (!ok) break;
            unsigned char *const from = base + Sh::kOffRing + slot * Sh::kStage;
#pragma unroll 1
            for (int step = 0; step < kStrips / W; ++step) {
                const int strip = warp * (kStrips / W) + step, key0 = first + tile * kTileKeys + step * kStrip;
                if (key0 >= kv1) break;
                const unsigned char *const ks = from + strip * KS, *const vs = ks + kStrips * KS;
                if (gone[slot] >> strip & 1) {  // on a page that the pool does not have: zeros
                    for (int i = lane; i < 32 * DG; i += 32)
                        reinterpret_cast<uint32_t *>(from + (i < 16 * DG ? 0 : kStrips * KS) + strip * KS + 256 * DG)[i % (16 * DG)] = 0;  // step and lo
                    smem_to_async();  // before the slot is loaded again
                    __syncwarp();
                }
                // S': lane has keys g and g + 8, rows 2 t and 2 t + 1 of each 8
                float s[NT][4];
                {
#pragma unroll
                    for (int i = 0; i < NT; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
                    uint32_t k0[DG], k1[DG], e0[DG], e1[DG];
                    words<DG>(ks + 16 * DG * g + 4 * DG * t, k0);
                    words<DG>(ks + 16 * DG * (g + 8) + 4 * DG * t, k1);
                    words<DG>(ks + 256 * DG + 4 * DG * g, e0);
                    words<DG>(ks + 256 * DG + 4 * DG * (g + 8), e1);
#pragma unroll
                    for (int j = 0; j < DG; ++j) {
                        uint32_t u[4], v[4];
                        values4<BF>(k0[j], low_twice(e0[j]), high_twice(e0[j]), u);
                        values4<BF>(k1[j], low_twice(e1[j]), high_twice(e1[j]), v);
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            uint4 q;
                            if constexpr (NT == 1) q = q1[j];
                            else q = qs[(i * DG + j) * 32 + lane];
                            product<BF>(s[i], u[0], v[0], u[1], v[1], q.x, q.y);
                            product<BF>(s[i], u[2], v[2], u[3], v[3], q.z, q.w);
                        }
                    }
                }
                const bool blind = key0 + kStrip > all_see;
                if (blind) {
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const int lim = sink.seen(8 * i + 2 * t + z) - key0 - g;
#pragma unroll
                            for (int y = 0; y < 2; ++y)
                                if (8 * y >= lim) s[i][2 * y + z] = -INFINITY;
                        }
                }
                float e[NT][4], over = -INFINITY;  // log2 of the weights, the highest of them
                const auto exponents = [&] {
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int z = 0; z < 4; ++z) e[i][z] = fmaf(s[i][z], c, off[i][z & 1]);
                };
                exponents();
#pragma unroll
                for (int i = 0; i < NT; ++i) over = max3(max3(over, e[i][0], e[i][1]), e[i][2], e[i][3]);
                if (__any_sync(FULL, over > kv_lift(BF) + kGrow)) {
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            float top = fmaxf(s[i][z], s[i][2 + z]);
#pragma unroll
                            for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(FULL, top, d));
                            if (fmaf(top, c, off[i][z]) > kv_lift(BF) + kGrow) {  // each row for itself: what it becomes does not hang on the rows beside it
                                const float to = kv_lift(BF) - top * c, f = ex2(to - off[i][z]);
                                off[i][z] = to;
                                sum[i][z] *= f;
#pragma unroll
                                for (int y = 0; y < 2 * DG; ++y) {
                                    o[i][y][z] *= f;
                                    o[i][y][2 + z] *= f;
                                }
                            }
                        }
                    exponents();
                }
                uint32_t p[NT][2];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
#pragma unroll
                    for (int z = 0; z < 4; ++z) s[i][z] = ex2(e[i][z]);
                    sum[i][0] += s[i][0] + s[i][2];
                    sum[i][1] += s[i][1] + s[i][3];
                    p[i][0] = turned(pack<BF>(s[i][0], s[i][1]));
                    p[i][1] = turned(pack<BF>(s[i][2], s[i][3]));
                }
                {
                    uint32_t v0[DG], v1[DG], f0[2 * DG], f1[2 * DG];
                    words<DG>(vs + 4 * DG * lane, v0);
                    words<DG>(vs + 128 * DG + 4 * DG * lane, v1);
                    words<2 * DG>(vs + 256 * DG + 8 * DG * t, f0);
                    words<2 * DG>(vs + 256 * DG + 8 * DG * (t + 4), f1);
                    if (blind) {  // values past the end of the keys, whatever they are, must not meet their zero probabilities
                        const int key = key0 + 2 * t;
                        const uint32_t m0 = (key < kv1 ? 0xffffu : 0u) | (key + 1 < kv1 ? 0xffff0000u : 0u);
                        const uint32_t m1 = (key + 8 < kv1 ? 0xffffu : 0u) | (key + 9 < kv1 ? 0xffff0000u : 0u);
#pragma unroll
                        for (int j = 0; j < DG; ++j) {
                            f0[2 * j] &= m0, f0[2 * j + 1] &= m0;
                            f1[2 * j] &= m1, f1[2 * j + 1] &= m1;
                            // Nor may a group that is not a number meet rows that do not see it: it is left out, and those that do are spoilt.
                            constexpr uint32_t kExp = BF ? 0x7f80u : 0x7c00u;
                            const auto odd = [&](const uint32_t *f, int half) {
                                const uint32_t st = f[2 * j] >> (16 * half), lo = f[2 * j + 1] >> (16 * half);
                                return (st & kExp) == kExp || (lo & kExp) == kExp;
                            };
                            const bool b0 = odd(f0, 0), b1 = odd(f0, 1), b2 = odd(f1, 0), b3 = odd(f1, 1);
                            if (__any_sync(FULL, b0 || b1 || b2 || b3)) {
                                const int least = __reduce_min_sync(FULL, b0 ? key : b1 ? key + 1 : b2 ? key + 8 : b3 ? key + 9 : INT_MAX);  // of such keys
                                const uint32_t n0 = (b0 ? 0u : 0xffffu) | (b1 ? 0u : 0xffff0000u), n1 = (b2 ? 0u : 0xffffu) | (b3 ? 0u : 0xffff0000u);
                                f0[2 * j] &= n0, f0[2 * j + 1] &= n0;
                                f1[2 * j] &= n1, f1[2 * j + 1] &= n1;
#pragma unroll
                                for (int i = 0; i < NT; ++i)
#pragma unroll
                                    for (int z = 0; z < 2; ++z)
                                        if (least < sink.seen(8 * i + 2 * t + z)) {
                                            o[i][2 * j][z] = o[i][2 * j][2 + z] = NAN;
                                            o[i][2 * j + 1][z] = o[i][2 * j + 1][2 + z] = NAN;
                                        }
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < DG; ++j) {
                        uint32_t u[4], v[4];
                        values4<BF>(v0[j], f0[2 * j], f0[2 * j + 1], u);
                        values4<BF>(v1[j], f1[2 * j], f1[2 * j + 1], v);
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            product<BF>(o[i][2 * j], u[0], u[1], v[0], v[1], p[i][0], p[i][1]);
                            product<BF>(o[i][2 * j + 1], u[2], u[3], v[2], v[3], p[i][0], p[i][1]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(empty(slot));
        }
        if (!ok) break;
        place(x + 1);
        float2 *const all_m = reinterpret_cast<float2 *>(base + Sh::kOffM + (x & 1) * Sh::kSizeM);
        // The warps' shares: columns 32 j + 4 g + (0 .. 3) of rows 2 t and 2 t + 1 of each 8.
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                float l = sum[i][z];
#pragma unroll
                for (int d = 4; d < 32; d *= 2) l += __shfl_xor_sync(FULL, l, d);
                if (g == 0) all_m[warp * R + 8 * i + 2 * t + z] = make_float2(off[i][z], l);
            }
        // What warp w's share of row y is multiplied by, in units of the one with the highest scores; the joint sum.
        const auto least = [&](int y) {
            float off = FLT_MAX;
#pragma unroll
            for (int w = 0; w < W; ++w) off = fminf(off, all_m[w * R + y].x);
            return off;
        };
        const auto factor = [&](int w, int y, float off) { return ex2(off - all_m[w * R + y].x); };
        const auto total_of = [&](int y, float off) {
            float total = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) total = fmaf(all_m[w * R + y].y, factor(w, y, off), total);
            return total;
        };
        float *const all_o = reinterpret_cast<float *>(base + Sh::kOffO);
#pragma unroll
        for (int i = 0; i < NT; ++i) {  // 8 rows at a time
            if (i > 0 && 8 * i >= rows) break;
            if (no > 0) ok = __all_sync(FULL, bar_wait(cleared, (no - 1) & 1, gave_up));  // the rows before have been read
            if (!ok) break;
            ++no;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                float *const to = all_o + (warp * 8 + 2 * t + z) * Sh::kPitch + 4 * g;
#pragma unroll
                for (int j = 0; j < DG; ++j)
                    *reinterpret_cast<float4 *>(to + 32 * j) = make_float4(o[i][2 * j][z], o[i][2 * j][2 + z], o[i][2 * j + 1][z], o[i][2 * j + 1][2 + z]);
            }
            join();
            if (!ok) break;
            for (int e = tid; e < min(rows - 8 * i, 8) * 8 * DG; e += 32 * W) {
                const int in = e / (8 * DG), y = 8 * i + in, d = e % (8 * DG) * 4;
                if (d >= D) continue;
                const float off0 = least(y), total = total_of(y, off0);
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float f = factor(w, y, off0);
                    const float4 u = *reinterpret_cast<const float4 *>(all_o + (w * 8 + in) * Sh::kPitch + d);
                    v = make_float4(fmaf(u.x, f, v.x), fmaf(u.y, f, v.y), fmaf(u.z, f, v.z), fmaf(u.w, f, v.w));
                }
                const typename Sink<BF, true>::Joint joint = sink.joint(-off0, total, sink.before(y));
                const float f = joint.mine, fb = joint.before;
                v = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
                float4 *const part = reinterpret_cast<float4 *>(a.part + (sg.row + y) * D + d);
                if (fb != 0.f) {
                    const float4 u = *part;
                    v = make_float4(fmaf(u.x, fb, v.x), fmaf(u.y, fb, v.y), fmaf(u.z, fb, v.z), fmaf(u.w, fb, v.w));
                }
                if (sg.direct) *reinterpret_cast<uint2 *>(sink.out_row(y) + d) = make_uint2(pack<BF>(v.x, v.y), pack<BF>(v.z, v.w));
                else *part = v;
            }
            __syncwarp();
            if (lane == 0) bar_arrive(cleared);
        }
        if (!ok) break;
        // the joint sums, once all have read the ones before
        if (sg.joins) join();
        if (!ok) break;
        for (int y = tid; y < rows; y += 32 * W) {
            const float off0 = least(y);
            sink.lse(y, sink.joint(-off0, total_of(y, off0), sink.before(y)).e);
        }
        __syncwarp();
        if (lane == 0) bar_arrive(seg_empty(x));
    }
    if (!ok && lane == 0) atomicMin(kv.status, SIM_E_STATE);
}

template <int DG, int NT, bool BF>
cudaError_t launch(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    constexpr int W = 4;
    using Sh = Shape<DG, NT, W>;
    static thread_local int ready = -1;  // the device on which the kernel has its shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev != ready) {
        e = cudaFuncSetAttribute((const void *)k_light_4bit<DG, NT, W, BF>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes);
        if (e == cudaSuccess) ready = dev;
    }
    return e == cudaSuccess ? launch_chained(k_light_4bit<DG, NT, W, BF>, kv_blocks(a.sms, 1, Sh::kPerSm), Sh::kThreads, Sh::kBytes, st, kv, b, a) : e;
}

template <int DG, bool BF>
cudaError_t launch_rows(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    return kv_light_rows(kv, b) == 8 ? launch<DG, 1, BF>(kv, b, a, st) : launch<DG, 2, BF>(kv, b, a, st);
}

template <bool BF>
cudaError_t launch_dims(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    switch (kv_dim_groups(kv)) {
        case 1: return launch_rows<1, BF>(kv, b, a, st);
        case 2: return launch_rows<2, BF>(kv, b, a, st);
        case 3: return launch_rows<3, BF>(kv, b, a, st);
        default: return launch_rows<4, BF>(kv, b, a, st);
    }
}

}  // namespace

cudaError_t launch_kv_light_4bit(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st) {
    return kv_bf(kv) ? launch_dims<true>(kv, b, a, st) : launch_dims<false>(kv, b, a, st);
}

}  // namespace simgb
