// Attention of heavy items (33 .. 256 query rows; see sim_kv_attend.cu), bound by the tensor products.
//
// One block per SM, two groups of four softmax warps with 128 rows each.  Both groups use every tile of 128 keys,
// so a byte that enters shared memory serves 256 rows; the tensor unit works for one group while the other is in its
// softmax (the second group rests while an item has at most 128 rows: 132 instead of 134 us for 64 sequences of 2048 keys with 128
// rows).  Per tile and group: S = Q K^T (128 x 128 x D, operands in shared memory), P = exp2(c (S - m)) written over
// S in TMEM as 16 bits, O += P V (128 x D x 128, P from TMEM, V as it lies, the N dimension contiguous).  TMEM is full:
// 128 columns each for S / P and O of the two groups.
//
// P is rounded to the cache's type (its relative error, 2^-9 or 2^-12, is that of the values it meets; in float16 with steps of
// 2^-31 below 2^-21, see kv_lift), its sum is not; m may lag behind the row's maximum by a factor of 2^kGrow before O is rescaled.
//
// 16 prompts' own 300 - 512 tokens on 4096 + 600 keys each, 64 heads, D = 128: 456 us, 1.69 PFLOP/s, 87 % of cuBLAS's
// burst rate.  A tile takes both groups about 2550 cycles, its products alone 2048.  In these, operands and loads ask shared
// memory for 256 KB (S 128, P V 64, the tile's arrival 64), which at 128 bytes a cycle is all that it can give; the rest is the
// way from a product through the softmax to the next one.  The first half of P is multiplied while the second is made (508 instead of 544 us, plan,
// light items and join included).
#include <type_traits>

#include "sim_kv_attend.cuh"

namespace simgb {

namespace {

constexpr int kPitch = 20;            // words between rows on the stage, 16 of them used: no bank conflicts
constexpr int kStage = 128 * kPitch;  // words through which the results of 128 rows pass

// The results of a warp's 32 rows from row0 on, 16 words of each at a time through `mine` (32 x kPitch words), so that stores
// fill sectors; what the lane's row is multiplied by, and what it has in the workspace (Sink::joint).
template <int DP, bool BF>
__device__ __forceinline__ void store_rows(const Sink<BF> &sink, uint32_t t_o, uint32_t *mine, int row0, int rows, float f, float fb) {
    const Segment &sg = sink.sg;
    const int lane = threadIdx.x & 31;
    char *to[4];  // this lane's 16 bytes of four rows
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int y = min(row0 + q * 8 + lane / 4, rows - 1);
        to[q] = (sg.direct ? reinterpret_cast<char *>(sink.out_row(y)) : reinterpret_cast<char *>(sink.a.part + (sg.row + y) * sink.D)) + lane % 4 * 16;
    }
    const int cols = sg.direct ? 32 : 16;
    const float *const old = sink.a.part + (sg.row + min(row0 + lane, rows - 1)) * sink.D;
    const auto add = [&](uint32_t *o, auto n, int d0) {
#pragma unroll
        for (int y = 0; y < decltype(n)::value; y += 4) {
            if (fb == 0.f || d0 + y >= sink.D) continue;
            const float4 v = *reinterpret_cast<const float4 *>(old + d0 + y);
            o[y] = __float_as_uint(fmaf(v.x, fb, __uint_as_float(o[y])));
            o[y + 1] = __float_as_uint(fmaf(v.y, fb, __uint_as_float(o[y + 1])));
            o[y + 2] = __float_as_uint(fmaf(v.z, fb, __uint_as_float(o[y + 2])));
            o[y + 3] = __float_as_uint(fmaf(v.w, fb, __uint_as_float(o[y + 3])));
        }
    };
#pragma unroll 1
    for (int d0 = 0; d0 < sink.D; d0 += cols) {
        uint32_t x[16];
        if (sg.direct) {
            uint32_t o[32];
            tm_ld32(t_o + d0, o);
            tc_wait_ld();
#pragma unroll
            for (int y = 0; y < 32; ++y) o[y] = f == 0.f ? 0 : __float_as_uint(__uint_as_float(o[y]) * f);
            if (sg.joins) add(o, std::integral_constant<int, 32>(), d0);
#pragma unroll
            for (int y = 0; y < 16; ++y) x[y] = pack<BF>(__uint_as_float(o[2 * y]), __uint_as_float(o[2 * y + 1]));
        } else {
            tm_ld16(t_o + d0, x);
            tc_wait_ld();
#pragma unroll
            for (int y = 0; y < 16; ++y) x[y] = f == 0.f ? 0 : __float_as_uint(__uint_as_float(x[y]) * f);
            if (sg.joins) add(x, std::integral_constant<int, 16>(), d0);
        }
#pragma unroll
        for (int y = 0; y < 16; y += 4) *reinterpret_cast<uint4 *>(mine + lane * kPitch + y) = make_uint4(x[y], x[y + 1], x[y + 2], x[y + 3]);
        __syncwarp();
        const bool in = d0 + lane % 4 * (cols / 4) < sink.D;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int y = q * 8 + lane / 4;
            const uint4 v = *reinterpret_cast<const uint4 *>(mine + y * kPitch + lane % 4 * 4);
            if (in && row0 + y < rows) *reinterpret_cast<uint4 *>(to[q]) = v;
            to[q] += 64;
        }
        __syncwarp();
    }
}

template <int DP>
struct Shape {
    static constexpr int kGroups = 2;
    static constexpr int kThreads = kGroups * 128 + 128;
    static constexpr int kTile = DP * 256;                                    // bytes of 128 query rows, or of a tile of keys or values
    static constexpr int kHalf = 16384;                                       // 128 rows of 64 columns
    static constexpr int kSlots = 131072 / kTile;                             // tiles of keys or values in flight
    static constexpr int kTmem = 512;
    static constexpr int kOffO = kGroups * 128;                               // TMEM column of the first group's O
    static constexpr int kSoftRegs = 208, kOtherRegs = 88;
    static_assert(kGroups * kSoftRegs + kOtherRegs <= (kGroups + 1) * 168, "the launch gives 168 registers a thread: no more are handed out");
    static constexpr int kOffRing = kGroups * kTile;
    static constexpr int kOffStage = kOffRing + kSlots * kTile;
    static constexpr int kOffSeg = kOffStage + kGroups * kStage * 4;
    // Keys with values that are not finite, in tiles that not all rows see whole, of segment x at x modulo twice kSegs: the warp
    // that finds them is less than that ahead of the softmax, without which no segment is told of kSegs later.
    static constexpr int kOffBad = kOffSeg + kSegs * int(sizeof(Segment));
    static constexpr int kOffBar = kOffBad + 2 * kSegs * kBlindTiles * 16;
    static constexpr int kBars = 2 * kSlots + 2 * kSegs + 2 + 4 * kGroups + 1 + kSlots;
    static constexpr int kBytes = kOffBar + kBars * 8 + 16;
    static constexpr int kAlloc = kBytes + 1024;                              // the base is rounded up to 1024
    static_assert(kAlloc <= 232448, "shared memory");
};

// A tile of 128 keys of the row in this thread's lane: S (columns t_s on) becomes P in 16 bits, in the same columns; half:
// called when its first half is in place.  lim: the last of the keys that the row sees.  m, l: the maximum that P refers to and
// the sum so far; DP columns of O from t_o on.
template <int DP, bool BF, typename Half>
__device__ __forceinline__ void softmax_tile(uint32_t t_s, uint32_t t_o, int lim, bool first, float c, float &m, float &l, Half &&half) {
    uint32_t s[kTileKeys];
#pragma unroll
    for (int q = 0; q < kTileKeys / 32; ++q) tm_ld32(t_s + 32 * q, s + 32 * q);
    tc_wait_ld();
    if (__any_sync(FULL, lim < kTileKeys - 1)) {
#pragma unroll
        for (int y = 0; y < kTileKeys; ++y)
            if (y > lim) s[y] = 0xff800000u;
    }
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int y = 0; y < kTileKeys; y += 2) top[y / 2 & 3] = max3(top[y / 2 & 3], __uint_as_float(s[y]), __uint_as_float(s[y + 1]));
    const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    if (first) {
        m = mx;
    } else if (const bool grows = (mx - m) * c > kGrow; __any_sync(FULL, grows)) {
        // each row for itself: what it becomes does not hang on the rows beside it, nor on what lies in lanes past the rows
        const float up = grows ? mx : m, f = grows ? ex2((m - up) * c) : 1.f;
        m = up;
        l *= f;
#pragma unroll 1
        for (int q = 0; q < DP / 32; ++q) {
            uint32_t o[32];
            tm_ld32(t_o + 32 * q, o);
            tc_wait_ld();
#pragma unroll
            for (int y = 0; y < 32; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * f);
            tm_st32(t_o + 32 * q, o);
        }
    }
    const float off = m == -INFINITY ? 0.f : m * c - kv_lift(BF);
    float2 sum[4] = {};
    uint32_t pk[kTileKeys / 2];
#pragma unroll
    for (int y = 0; y < kTileKeys; y += 2) {
        float2 e = fma2(make_float2(__uint_as_float(s[y]), __uint_as_float(s[y + 1])), make_float2(c, c), make_float2(-off, -off));
        e = make_float2(ex2(e.x), ex2(e.y));
        sum[y / 2 & 3] = add2(sum[y / 2 & 3], e);
        pk[y / 2] = pack<BF>(e.x, e.y);
        if (y == kTileKeys / 2 - 2) {
            tm_st32(t_s, pk);
            tc_wait_st();
            half();
        }
    }
    sum[0] = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
    l += sum[0].x + sum[0].y;
    tm_st32(t_s + 32, pk + 32);
    tc_wait_st();
}

template <int DP, bool BF>
__global__ void __launch_bounds__(Shape<DP>::kThreads, 1)
    k_heavy(const sim_kv kv, const sim_kv_batch b, const KvAttend a, const __grid_constant__ KvMaps maps) {
    using Sh = Shape<DP>;
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
    const auto p_half = [&](int g) { return bars + 8 * (kRest + 2 + 3 * NG + g); };
    const uint32_t drained = bars + 8 * (kRest + 2 + 4 * NG);
    // The x-th tile of values that is looked at is being loaded (only from then on can one wait for it to be there); has been looked
    // at.  No more than NS / 2 are loaded that are not yet multiplied.
    const auto look_at = [&](uint32_t x) { return bars + 8 * (kRest + 3 + 4 * NG + x % (NS / 2)); };
    const auto clean = [&](uint32_t x) { return bars + 8 * (kRest + 3 + 4 * NG + NS / 2 + x % (NS / 2)); };
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
            bar_init(p_half(g), 4);
            bar_init(o_full(g), 2);
        }
        bar_init(drained, 1);
        for (int x = 0; x < NS / 2; ++x) {
            bar_init(look_at(x), 1);
            bar_init(clean(x), 2);
        }
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 128 * NG) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.keys) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.values) : "memory");
        if (maps.q_boxes) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.queries) : "memory");
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
            Line line(plan, kv.n_kv_heads, 0, blockIdx.x, a.sms);
            const int P = kv.page_size, per = kTileKeys / P;
            uint32_t at = 0, nc = 0;  // tiles loaded, those looked at
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
                const int clean_from = Sink<BF>{kv, a, sg, G, D, b.q_heads}.clean_from();
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
                    for (int v = 0; v < 2; ++v, ++at) {  // keys, values
                        ok = __all_sync(FULL, bar_wait(empty(at), (at / NS + 1) & 1, gave_up));
                        if (!ok) break;
                        if (lane == 0) bar_expect(full(at), Sh::kTile);
                        __syncwarp();
                        if (lane < per) {
                            const uint32_t dst = sbase + Sh::kOffRing + (at % NS) * Sh::kTile + lane * P * 128;
#pragma unroll
                            for (int half = 0; half < DP / 64; ++half)
                                tma_load(dst + half * Sh::kHalf, v ? &maps.values : &maps.keys, full(at), half * 64, 0, sg.h, w);
                        }
                    }
                    if (ok && j >= clean_from) {
                        if (lane == 0) bar_arrive(look_at(nc));
                        ++nc;
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
            uint32_t at = 0, nc = 0, np[NG] = {};
            bool ok = true;
            const auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(FULL, bar_wait(bar, parity, gave_up)) != 0; };
            const auto wait_full = [&](uint32_t y) { return wait(full(y), (y / NS) & 1); };
            Segment sg;
            for (uint32_t x = 0; (ok = take(x, sg)); ++x) {
                const int n = __shfl_sync(FULL, sg.n, 0), last = __shfl_sync(FULL, sg.rows, 0) > 128;  // group with rows
                if (n == 0) break;
                const int clean_from = __shfl_sync(FULL, Sink<BF>{kv, a, sg, G, D, b.q_heads}.clean_from(), 0);
                const auto keys = [&](int j, int g) {  // S of group g and tile j
                    if (elect_one()) {
                        const uint32_t slot = (at + 2 * j) % NS;
#pragma unroll
                        for (int kk = 0; kk < DP / 16; ++kk) {
                            const uint32_t off = (kk / 4) * Sh::kHalf + (kk % 4) * 32;
                            mma_ss(tmem + g * 128, op_q + ((g * Sh::kTile + off) >> 4), op_k + ((slot * Sh::kTile + off) >> 4), idesc_s, kk > 0);
                        }
                        tc_commit(s_full(g));
                        if (g == last) {
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
                for (int g = 0; g < NG; ++g)
                    if (g <= last) keys(0, g);
                for (int j = 0; j < n && ok; ++j) {
                    ok = wait_full(at + 2 * j + 1);
                    if (ok && j >= clean_from) ok = wait(clean(nc), nc / (NS / 2) & 1), ++nc;
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        if (g > last) break;
                        const uint32_t slot = (at + 2 * j + 1) % NS;
                        const auto values = [&](int from) {  // half of the tile's keys
                            tc_fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int kk = 0; kk < kTileKeys / 32; ++kk)
                                    mma_ts(tmem + Sh::kOffO + g * 128, tmem + g * 128 + (from + kk) * 8, op_v + ((slot * Sh::kTile + (from + kk) * 2048) >> 4), idesc_o, j > 0 || from + kk > 0);
                                if (from > 0) {
                                    if (g == last) tc_commit(empty(at + 2 * j + 1));
                                    if (j + 1 == n) {
                                        tc_commit(o_full(g));
                                        bar_arrive(o_full(g));  // what the look at the values has found is in shared memory
                                    }
                                }
                            }
                            __syncwarp();
                        };
                        ok = ok && wait(p_half(g), np[g] & 1);
                        if (!ok) break;
                        values(0);
                        ok = wait(p_ready(g), np[g]++ & 1);
                        if (!ok) break;
                        values(kTileKeys / 32);
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
            // ---- query rows, by TMA where heads and tokens make boxes of 128 rows (rows of other entries, past the item's,
            // come with them); else two warps, 16 bytes a lane, the lanes of a row side by side (all that prefill 532 instead of
            // 508 us).  What rows past the item's hold meets no other row and is not used.
            // They then look at the values of the item's last tiles, before they are multiplied: those past the end of
            // the keys, whatever they are, must not meet their zero probabilities, nor those that are not finite the rows that do not
            // see them (by the softmax's warps instead: 531 us).
            constexpr int kVec = DP / 8, kStep = 64 / kVec;
            const int j = (tid & 63) % kVec;
            const bool has = j * 8 < D;
            const auto look = [&](const Segment &s, uint32_t x, uint32_t at, uint32_t &nc) {
                const Sink<BF> sink = {kv, a, s, G, D, b.q_heads};
                const int blind_from = sink.blind_from();
                uint32_t *const bad = reinterpret_cast<uint32_t *>(base + Sh::kOffBad) + x % (2 * kSegs) * kBlindTiles * 4;
                for (int t = sink.clean_from(); t < s.n; ++t, ++nc) {
                    const uint32_t y = at + 2 * t + 1;
                    if (!__all_sync(FULL, bar_wait(look_at(nc), nc / (NS / 2) & 1, gave_up) && bar_wait(full(y), (y / NS) & 1, gave_up))) return false;
#pragma unroll 1
                    for (int r = (role - 2) * 64 + lane; r < (role - 1) * 64; r += 32) {
                        unsigned char *const v = base + Sh::kOffRing + (y % NS) * Sh::kTile + r * 128;
                        bool found = false;
                        if (r >= s.kv1 - s.k0 - t * kTileKeys) {
#pragma unroll
                            for (int z = 0; z < DP / 8; ++z) *reinterpret_cast<uint4 *>(v + (z / 8) * Sh::kHalf + (z % 8) * 16) = make_uint4(0, 0, 0, 0);
                        } else if (t >= blind_from) {
                            found = clean_row<DP, BF>(v, Sh::kHalf);
                        }
                        const unsigned keys = __ballot_sync(FULL, found);
                        if (t >= blind_from && lane == 0) bad[(t - blind_from) * 4 + r / 32] = keys;
                    }
                    smem_to_async();
                    __syncwarp();
                    if (lane == 0) bar_arrive(clean(nc));
                }
                return true;
            };
            Segment sg;
            uint32_t x = 0, at = 0, nc = 0;
            for (; take(x, sg) && sg.n > 0; ++x) {
                if (!__all_sync(FULL, bar_wait(q_empty, (x + 1) & 1, gave_up))) break;
                if (maps.q_boxes) {
                    if (lane == 0) {
                        if (role == 2) {
                            const int ng = sg.rows > 128 ? NG : 1;
                            bar_expect(q_full, ng * Sh::kTile);
                            for (int g = 0; g < ng; ++g)
                                for (int half = 0; half < DP / 64; ++half)
                                    tma_load3(sbase + g * Sh::kTile + half * Sh::kHalf, &maps.queries, q_full, half * 64, sg.h * G, sg.q0 + a.group.div(sg.row0 + g * 128));
                        } else {
                            bar_arrive(q_full);
                        }
                    }
                    __syncwarp();
                    if (!look(sg, x, at, nc)) break;
                    at += 2 * sg.n;
                    continue;
                }
                const uint16_t *const from0 = static_cast<const uint16_t *>(a.q) + int64_t(sg.q0) * a.qt + int64_t(sg.h * G) * a.qh + (has ? j * 8 : 0);
#pragma unroll 4
                for (int r = (tid & 63) / kVec; r < sg.rows; r += kStep) {
                    const int y = sg.row0 + r, t = a.group.div(y);
                    const uint16_t *from = from0 + int64_t(t) * a.qt + int64_t(y - t * G) * a.qh;
                    const uint32_t to = sbase + (r >> 7) * Sh::kTile + (j / 8) * Sh::kHalf + (r & 127) * 128 + (((j % 8) ^ (r & 7)) << 4);
                    if (a.q_vec) {
                        const int bytes = has ? 16 : 0;  // columns past the head's are zeros
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
                    } else {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (has)
                            v = make_uint4(from[0] | uint32_t(from[1]) << 16, from[2] | uint32_t(from[3]) << 16, from[4] | uint32_t(from[5]) << 16,
                                           from[6] | uint32_t(from[7]) << 16);
                        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                smem_to_async();
                __syncwarp();
                if (lane == 0) bar_arrive(q_full);
                if (!look(sg, x, at, nc)) break;
                at += 2 * sg.n;
            }
            // after a wait that gave up: the last boxes may be on their way
            if (maps.q_boxes && x > 0)
                for (int n = 0; n < 1000000 && *gave_up && !bar_try(q_full, (x - 1) & 1); ++n) {
                }
        }
    } else {
        // ---- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kSoftRegs));
        const int g = warp >> 2, w = warp & 3, lr = tid & 127;
        const uint32_t t_lane = tmem + (uint32_t(w * 32) << 16), t_s = t_lane + g * 128, t_o = t_lane + Sh::kOffO + g * 128;
        uint32_t *const stage = reinterpret_cast<uint32_t *>(base + Sh::kOffStage) + g * kStage;
        const float c = a.scale_log2;
        uint32_t ns = 0, no = 0;
        bool ok = true;
        Segment sg;
        for (uint32_t x = 0; ok && take(x, sg) && sg.n > 0; ++x) {
            if (sg.rows <= g * 128) continue;
            const int r = g * 128 + lr;  // the row in this thread's lane
            // key position that it sees last; lanes past the rows see all: theirs are no reason to mask a tile
            const int last = r < sg.rows ? min(sg.kv1 - 1, sg.pos0 + int(a.group.div(sg.row0 + r))) : sg.kv1 - 1;
            const Sink<BF> sink = {kv, a, sg, G, D, b.q_heads};
            const int blind_from = sink.blind_from();
            const uint32_t *const bad = reinterpret_cast<const uint32_t *>(base + Sh::kOffBad) + x % (2 * kSegs) * kBlindTiles * 4;
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < sg.n; ++j) {
                const int k0 = sg.k0 + j * kTileKeys;  // first key of the tile
                ok = __all_sync(FULL, bar_wait(s_full(g), ns & 1, gave_up));
                if (!ok) break;
                ++ns;
                tc_fence_after();
                softmax_tile<DP, BF>(t_s, t_o, last - k0, j == 0, c, m, l, [&] {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_half(g));
                });
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_ready(g));
            }
            if (!ok) break;
            const typename Sink<BF>::Joint joint = sink.joint(m * c - kv_lift(BF), l, r < sg.rows ? sink.before(r) : -INFINITY);
            if (r < sg.rows) sink.lse(r, joint.e);
            ok = __all_sync(FULL, bar_wait(o_full(g), no++ & 1, gave_up));
            if (!ok) break;
            tc_fence_after();
            store_rows<DP>(sink, t_o, stage + w * 32 * kPitch, r - lane, sg.rows, joint.mine, joint.before);
            uint32_t some = 0;
#pragma unroll 1
            for (int z = 0; z < 4 * (sg.n - blind_from); ++z) some |= bad[z];
            if (some)
                for (int y = r - lane; y < min(r - lane + 32, sg.rows); ++y) sink.spoil(y, bad);
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

template <int DP, bool BF>
cudaError_t launch(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, const KvMaps &maps, cudaStream_t st) {
    static thread_local int ready = -1;  // the device on which the kernel has its shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev != ready) {
        e = cudaFuncSetAttribute((const void *)k_heavy<DP, BF>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP>::kAlloc);
        if (e == cudaSuccess) ready = dev;
    }
    // queries by TMA: 128 rows are 128 / G tokens of G heads
    KvMaps m = maps;
    const uint32_t G = uint32_t(b.q_heads / kv.n_kv_heads);
    if (a.q_vec && 128 % G == 0 && a.qt > 0 && a.qh > 0) {
        const uint64_t dim[3] = {uint64_t(kv.head_dim), uint64_t(b.q_heads), uint64_t(b.n_q)}, stride[2] = {uint64_t(a.qh) * 2, uint64_t(a.qt) * 2};
        const uint32_t box[3] = {64, G, 128 / G};
        m.q_boxes = kv_encode_map(kv, &m.queries, 3, a.q, dim, stride, box);
    }
    return e == cudaSuccess ? launch_chained(k_heavy<DP, BF>, kv_blocks(a.sms, 0), Shape<DP>::kThreads, Shape<DP>::kAlloc, st, kv, b, a, m) : e;
}

}  // namespace

cudaError_t launch_kv_heavy(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, const KvMaps &maps, cudaStream_t st) {
    if (kv.dtype == SIM_KV_BF16) return kv.head_dim > 64 ? launch<128, true>(kv, b, a, maps, st) : launch<64, true>(kv, b, a, maps, st);
    return kv.head_dim > 64 ? launch<128, false>(kv, b, a, maps, st) : launch<64, false>(kv, b, a, maps, st);
}

}  // namespace simgb
