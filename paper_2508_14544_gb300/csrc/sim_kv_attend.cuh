// Device code shared by the attention kernels over the paged cache (sim_kv_attend.cu, sim_kv_heavy.cu, sim_kv_light.cu).
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include <climits>
#include <cmath>

#include "sim.h"
#include "sim_kv_internal.h"

namespace simgb {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int kSegs = 4;      // segments that the loading warp may be ahead
// Tiles that a segment has at most; longer stretches of an item are several segments, each of which adds to what the last has left
// in the workspace.  The tensor products' sums are cut off, not rounded, after every 16 keys: sums of one sign lose 2^-24 of
// themselves each time, 2^-13 in all over 256 tiles (over 10^6 keys, 0.6 %; the joining is rounded).  It also bounds how long the
// warps of a block wait for each other.  Taking up a segment costs some 4 tiles.
constexpr int kMostTiles = 256;
constexpr float kGrow = 8.f;  // log2 of what P may reach before O is rescaled
// log2 of what P, and the sum that its product is divided by, are multiplied by: up to 2^15, float16 has room, and below 2^-14 it
// has fewer and fewer bits.  So a key keeps all of its bits of P down to 2^-21 of the largest one's, and some down to 2^-32; many
// small weights beside a large one are not lost (32767 of 2^-25 are 2^-10 in all).
__host__ __device__ constexpr float kv_lift(bool bf) { return bf ? 0.f : 7.f; }

// A list's line (the spans of its items, one after the other) divided among its blocks: [at(c), at(c + 1)) is block c's,
// each + 1 places for the first `rest` blocks and `each` for the others.
struct Share {
    int64_t units, each;
    int rest;
    __device__ Share(int64_t units_, int blocks) : units(units_) {
        each = units_ <= INT_MAX ? int64_t(uint32_t(units_) / uint32_t(blocks)) : units_ / blocks;
        rest = int(units - each * blocks);
    }
    __device__ Share(const KvPlan &p, int light) {
        const int32_t *h = p.hdr + 16 * light;
        units = *reinterpret_cast<const int64_t *>(h + 2);
        each = *reinterpret_cast<const int64_t *>(h + 4);
        rest = h[6];
    }
    __device__ int64_t at(int c) const { return each * c + min(c, rest); }
    __device__ int of(int64_t u) const {  // the block that has place u < units
        const int64_t more = (each + 1) * rest;
        const bool front = u < more;
        const int64_t n = front ? u : u - more, d = front ? each + 1 : each;
        const int c = n <= INT_MAX && d <= INT_MAX ? int(uint32_t(n) / uint32_t(d)) : int(n / d);
        return front ? c : rest + c;
    }
};

// First row of the partial results of block c's piece of a list whose rows follow `base` others.
__device__ __forceinline__ int64_t piece_row(const KvItem &it, int h, int c, int64_t base, int light) {
    return base + it.row_off + int64_t(h) * it.rows + int64_t(kv_rows(light)) * c;
}
__device__ __forceinline__ int64_t list_base(const KvPlan &p, int light, int sms) {
    return light ? *reinterpret_cast<const int64_t *>(p.hdr + 24) + int64_t(kAttRows) * kv_blocks(sms, 0) : 0;
}

// A stretch of one item and kv head, as the warps of a block pass it on.
struct alignas(16) Segment {
    int32_t n;               // tiles, 0: the end
    int32_t h;
    int32_t q0, row0, rows, pos0;
    int32_t k0, kv1;         // first key, end of the keys
    int32_t seq;             // row of the table
    bool direct;             // results go to the output, not to the workspace
    bool joins;              // what the workspace has in that place is part of them
    int64_t row;             // row of the partial results
};

// Walks the stretch of a list's line that is block c's.
struct Line {
    const KvItem *items;
    KvItem it;
    int64_t u, u1, base;
    int n_items, heads, k, h, c, light;
    int t, t_end, whole;  // tiles of the item and head that are left, and whether all of them are this block's
    __device__ Line(const KvPlan &p, int heads_, int light_, int c_, int sms) : items(p.items[light_]), heads(heads_), c(c_), light(light_) {
        n_items = p.hdr[16 * light];
        const Share share(p, light);
        u = share.at(c);
        u1 = share.at(c + 1);
        base = list_base(p, light, sms);
        k = p.start[light][c];
        h = -1;
        t = t_end = whole = 0;
    }
    // The next item and head with work for this block; s.n = 0 at the end.
    __device__ void next(Segment &s) {
        s.n = 0;
        if (t < t_end) return part(s, true);
        while (u < u1 && k < n_items) {
            if (h < 0) it = items[k];
            const int span = kv_span(it.tiles, light);
            if (span == 0 || h + 1 == heads) {
                ++k;
                h = -1;
                continue;
            }
            h = h < 0 ? int(uint32_t(u - it.unit) / uint32_t(span)) : h + 1;
            const int64_t a = it.unit + int64_t(h) * span, tile0 = a + kv_lead(light);
            t = int(max(u - tile0, int64_t(0)));
            t_end = int(min(u1 - tile0, int64_t(it.tiles)));
            whole = t_end - t == it.tiles && !it.partial;
            u = a + span;
            if (t < t_end) return part(s, false);
        }
    }
    __device__ void part(Segment &s, bool joins) {
        s.n = min(t_end - t, kMostTiles);
        s.h = h;
        s.q0 = it.q0;
        s.row0 = it.row0;
        s.rows = it.rows;
        s.pos0 = it.pos0;
        s.k0 = it.kv0 + t * kTileKeys;
        s.kv1 = it.kv1;
        s.seq = it.seq;
        t += s.n;
        s.direct = whole && t == t_end;
        s.joins = joins;
        s.row = piece_row(it, h, c, base, light);
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

__device__ __forceinline__ void tma_load3(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map),
        "r"(bar), "r"(x), "r"(y), "r"(z)
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
__device__ __forceinline__ void tm_ld8(uint32_t addr, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : REG4(r, 0), REG4(r, 4) : "r"(addr));
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        VAL4(r, 0), VAL4(r, 4), VAL4(r, 8), VAL4(r, 12), VAL4(r, 16), VAL4(r, 20), VAL4(r, 24), VAL4(r, 28)
        : "memory");
}
__device__ __forceinline__ void tm_st8(uint32_t addr, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), VAL4(r, 0), VAL4(r, 4) : "memory");
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

// A row meets the values of a tile's keys that it does not see with probability 0, which is not nothing where they are infinite
// or not a number.  In tiles that some rows do not see whole (Sink::blind_from), each key's values (`row`, and `half` bytes on
// the next 64 columns) are looked at before the product, one fused multiply-add for two, and those that are not finite become
// zeros; Sink::spoil gives the rows that do see them their due.  True if the key has such values.  An item of 256 rows has three
// of these tiles at most, a single token none.
constexpr int kBlindTiles = 3;
template <int DP, bool BF>
__device__ __forceinline__ bool clean_row(unsigned char *row, int half) {
    const int turn = threadIdx.x & 7;  // 8 lanes, 8 places of 16 bytes: no bank conflicts
    uint32_t sum[4] = {};              // of 0 times the values: not 0 if one is not finite
    const auto fma0 = [](uint32_t x, uint32_t &y) {
        if (BF) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(y) : "r"(x), "r"(0));
        else asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(y) : "r"(x), "r"(0));
    };
#pragma unroll
    for (int z = 0; z < DP / 8; ++z) {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + z / 8 * half + (z % 8 ^ turn) * 16);
        fma0(v.x, sum[0]);
        fma0(v.y, sum[1]);
        fma0(v.z, sum[2]);
        fma0(v.w, sum[3]);
    }
    if (!((sum[0] | sum[1] | sum[2] | sum[3]) & 0x7fff7fffu)) return false;
    constexpr uint32_t kExp = BF ? 0x7f80u : 0x7c00u;
#pragma unroll 1
    for (int z = 0; z < DP / 2; ++z) {
        uint32_t *const at = reinterpret_cast<uint32_t *>(row + z / 32 * half) + z % 32;
        uint32_t w = *at;
        if ((w & kExp) == kExp) w &= 0xffff0000u;
        if ((w >> 16 & kExp) == kExp) w &= 0xffffu;
        *at = w;
    }
    return true;
}

// Where the results of a segment go.
template <bool BF>
struct Sink {
    const sim_kv &kv;
    const KvAttend &a;
    const Segment &sg;
    int G, D, q_heads;
    // First key of the segment that row y does not see.
    __device__ int seen(int y) const { return min(sg.kv1, sg.pos0 + int(a.group.div(sg.row0 + y)) + 1); }
    // The first tile that row 0, which sees the fewest keys, does not see as far as the item's keys go; sg.n: none.
    __device__ int blind_from() const {
        const int none = seen(0);
        return none < min(sg.kv1, sg.k0 + sg.n * kTileKeys) ? max(none - sg.k0, 0) / kTileKeys : sg.n;
    }
    // The first tile whose values are looked at before the product: a blind one, or one past the end of the keys; sg.n: none.
    __device__ int clean_from() const { return min(blind_from(), sg.kv1 - (sg.k0 + (sg.n - 1) * kTileKeys) < kTileKeys ? sg.n - 1 : sg.n); }
    // A row that sees values which clean_row took for zeros: its result in their columns is what they alone add up to, infinite
    // or not a number.  bad: a bit for each key of the tiles from blind_from on.  By one warp, a lane for four columns.
    __device__ void spoil(int y, const uint32_t *bad) const {
        const int lane = threadIdx.x & 31, P = kv.page_size, d = 4 * lane, from = blind_from(), stop = seen(y);
        const uint16_t *values = static_cast<const uint16_t *>(kv.pool) + a.layer * kv_layer_elems(kv) + kv_layer_elems(kv) / 2;
        float o[4] = {};
#pragma unroll 1
        for (int z = 0; z < 4 * (sg.n - from); ++z) {
            const int key = sg.k0 + from * kTileKeys + z * 32 + lane;
            int64_t at = -1;
            if ((bad[z] >> lane & 1) && key < stop) {
                const int page = kv.table[int64_t(sg.seq) * kv.max_pages + key / P];
                if (unsigned(page) < unsigned(kv.n_pages)) at = page * (kv_page_bytes(kv) / 2) + (int64_t(sg.h) * P + key % P) * D;
            }
            if (!__any_sync(FULL, at >= 0)) continue;
#pragma unroll 4
            for (int k = 0; k < 32; ++k) {
                const int64_t ak = __shfl_sync(FULL, at, k);
                const uint2 v = ak >= 0 && d < D ? *reinterpret_cast<const uint2 *>(values + ak + d) : make_uint2(0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint16_t bits = uint16_t((i < 2 ? v.x : v.y) >> i % 2 * 16);
                    const float x = BF ? __uint_as_float(uint32_t(bits) << 16) : __half2float(__ushort_as_half(bits));
                    if (x * 0.f != 0.f) o[i] += x;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (o[i] == 0.f) continue;
            if (sg.direct) out_row(y)[d + i] = uint16_t(pack<BF>(o[i], o[i]));
            else a.part[(sg.row + y) * D + d + i] = o[i];
        }
    }
    __device__ uint16_t *out_row(int y) const {  // of row y of the item
        const int t = a.group.div(sg.row0 + y);
        return static_cast<uint16_t *>(a.out) + int64_t(sg.q0 + t) * a.ot + int64_t(sg.h * G + (sg.row0 + y - t * G)) * a.oh;
    }
    // What row y's result over this segment, before the division by `total`, and the one in the workspace are multiplied by to
    // make up the joint one; log2 of the joint sum of exponentials, where `top` is log2 of what `total` is in units of.
    struct Joint {
        float mine, before, e;
    };
    __device__ float before(int y) const { return sg.joins ? a.part_lse[sg.row + y] : -INFINITY; }  // log2 of the sum so far
    __device__ Joint joint(float top, float total, float before) const {
        Joint x = {total == 0.f ? 0.f : 1.f / total, 0.f, total == 0.f ? -INFINITY : top + log2f(total)};
        if (before != -INFINITY) {
            const float up = fmaxf(x.e, before), mine = x.e == -INFINITY ? 0.f : ex2(x.e - up), old = ex2(before - up), f = 1.f / (mine + old);
            x = {x.mine * mine * f, old * f, up + log2f(mine + old)};
        }
        return x;
    }
    __device__ void lse(int y, float e) const {  // log2
        if (!sg.direct) {
            a.part_lse[sg.row + y] = e;
        } else if (a.lse) {
            const int t = a.group.div(sg.row0 + y);
            a.lse[int64_t(sg.q0 + t) * q_heads + sg.h * G + (sg.row0 + y - t * G)] = e * 0.69314718055994531f;
        }
    }
};

}  // namespace

// Tensor maps of one layer's keys and values, [page][head][token][dim], with boxes of the tokens of one
// page and head and 64 columns; of the queries [token][head][dim], with boxes of 128 rows (if q_boxes).
struct KvMaps {
    CUtensorMap keys, values, queries;
    int q_boxes;
};
// 16-bit floats of kv.dtype; strides in bytes from the second dimension on.  False if the driver refuses.
bool kv_encode_map(const sim_kv &kv, CUtensorMap *map, int rank, const void *at, const uint64_t *dim, const uint64_t *stride, const uint32_t *box);
cudaError_t launch_kv_heavy(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, const KvMaps &maps, cudaStream_t st);
cudaError_t launch_kv_light(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, const KvMaps &maps, cudaStream_t st);

}  // namespace simgb
