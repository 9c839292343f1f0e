// Keys and values of a 4-bit cache: quantised as they are written, and read back (16-bit caches are read here too).
//   k_write_4bit - bound by arithmetic: some 19 instructions a value (the difference from the lowest, its quotient to the nearest float, that to
//                the nearest whole number, 4 bits into their place; a third is what a group costs), 2.9 a cycle and SM.  343 us for
//                524 million values, of which HBM needs 204; 5.6 us for 40 tokens, a chain of two loads and the arithmetic.  The way
//                there, each from the one before: a thread for each group, its pieces stored apart 958 us, and 45
//                sectors written for a token's keys of a head instead of 4; by warps 637; each lane the step of one group instead of all
//                lanes those of all 385; differences checked by two roundings only where -lo lies next to a border 370; one row at a time,
//                so that four blocks fit 343.
//   k_read     - bound by HBM: 151 us for 0.95 GB, 6.3 TB/s; 6 us for a few tokens, a chain of dependent loads (offsets, entry, page, strip).
//                Of a 16-bit cache 277 us for 1.57 GB, 5.7 TB/s: what a lane keeps until it stores takes 128 registers, so that two blocks
//                fit an SM.  Every block walks the whole list of offsets to see that they are in order, which is nothing for the
//                lists of a batch (1500 entries: as fast as 1000) and most of the time of long ones: 10^5 entries of three tokens 1.8 ms
//                (16 bits: 2.3), of which their rows need 0.2 and 0.36.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "sim.h"
#include "sim_kv_4bit.cuh"

namespace simgb {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int kWrite = 256, kRead = 256;  // threads
constexpr int kFewEntries = 1024;

template <bool BF>
__device__ __forceinline__ float wide(uint32_t x, int half) {
    if (BF) return __uint_as_float(half ? x & 0xffff0000u : x << 16);
    const __half2 h = *reinterpret_cast<const __half2 *>(&x);
    return half ? __high2float(h) : __low2float(h);
}
template <bool BF>
__device__ __forceinline__ float wide16(uint32_t bits) {
    return BF ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half(uint16_t(bits)));
}
template <bool BF>
__device__ __forceinline__ uint32_t min16(uint32_t a, uint32_t b) {
    uint32_t d;
    if (BF) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <bool BF>
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
    uint32_t d;
    if (BF) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// The largest 16-bit float that is not above (hi - lo) / 15, as bits.  A product with slightly less than 1 / 15, cut off, gives it or the
// one below; 15 times a 16-bit float is a 32-bit one, so that comparing it with the difference, cut off too, is exact.
template <bool BF>
__device__ __forceinline__ uint32_t step_of(float lo, float hi) {
    // a difference past the largest float: of an eighth of both, which is exact but for what is far below the last place
    const bool large = BF && (hi > 1e38f || lo < -1e38f);
    const float span = large ? __fsub_rz(hi * 0.125f, lo * 0.125f) : __fsub_rz(hi, lo), q = __fmul_rz(span, 0x1.11111p-4f);
    uint32_t step, up;
    if (BF) {
        step = __float_as_uint(q) >> 16;
        up = step + 1;
        step = 15.f * __uint_as_float(up << 16) <= span ? up : step;
        if (large && step) step += 3 << 7;  // (a span of 0 has no step)
    } else {
        step = __half_as_ushort(__float2half_rz(q));
        up = step + 1;
        step = 15.f * __half2float(__ushort_as_half(uint16_t(up))) <= span ? up : step;
    }
    return step == 0 && hi > lo ? 1 : step;
}

// Next to a border between two codes, (k + 1/2) s, r = (x - lo) / s decides only which one: then t = x - lo, as a 32-bit float, and
// the rest are compared with the border, which is exact.
__device__ __forceinline__ float code_at_border(float x, float lo, float t, float r, float s) {
    const float k = floorf(r), border = fmaf(k, s, 0.5f * s);
    // t + rest = x - lo exactly (a sum of two floats and its rounding error)
    const float y = t - x, rest = (x - (t - y)) + (-lo - y);
    const bool tie = t == border && rest == 0.f;
    const bool up = tie ? int(k) & 1 : t == border ? rest > 0.f : t > border;
    return k + (up ? 1.f : 0.f);
}

// Codes of eight values, place q of them at the bits that the powers of two in `at` give: any values of the type, lo the lowest of
// the group and s its step.
template <bool BF>
__device__ __noinline__ uint32_t codes_exactly(uint4 x, float lo, float s, bool by_column) {
    // Tiny steps, whose reciprocals overflow, and large ones, whose differences do, after a multiplication by a power of two.
    const float more = BF && s < 0x1p-60f ? 0x1p60f : BF && s > 0x1p110f ? 0x1p-8f : 1.f;
    s *= more;
    lo *= more;
    const float inv = 1.f / s;
    uint32_t w = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const uint32_t pair = q < 2 ? x.x : q < 4 ? x.y : q < 6 ? x.z : x.w;
        const float val = wide<BF>(pair, q % 2) * more, t = val - lo, r = t * inv;  // r: within 2^-20 of the quotient, where it is below 16
        float code = rintf(r);
        if (fabsf(r - code) > 0.5f - 0x1p-18f) code = code_at_border(val, lo, t, r, s);
        w |= uint32_t(fminf(code, 15.f)) << (by_column ? 4 * q : 4 * (q / 2) + 16 * (q % 2));
    }
    return w;
}

// A warp for 16 tokens' keys, or values, of a head, one after the other; lane 4 g + t has columns 8 t .. 8 t + 7 of each group of tokens g and g + 8.
// Where 16 tokens of the list fill a strip, it is put together in shared memory and stored by 16 bytes; others' pieces are stored
// each for itself (a list's tokens lie on strips in any way, but those of a prompt fill most that they touch).
// VEC: the sources are 16-byte aligned.
template <int DG, bool BF, bool VEC>
__global__ void __launch_bounds__(kWrite, 4) k_write_4bit(const sim_kv kv, const KvWrite a, int each, int few) {
    __shared__ __align__(16) unsigned char images[kWrite / 32][320 * DG];
    kv_wait_previous();
    const int P = kv.page_size, D = kv.head_dim, H = kv.n_kv_heads, shift = __ffs(P) - 1, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    unsigned char *const image = images[threadIdx.x >> 5];
    // A warp takes `each` of a chunk's heads; of few tokens, one head's 8 of the 16, whatever they fill.
    const int parts = few ? 4 * H : (2 * H + each - 1) / each;
    const int64_t jobs = (int64_t(a.n_new) + kStrip - 1) / kStrip * parts;
    for (int64_t job = int64_t(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5); job < jobs; job += int64_t(gridDim.x) * (blockDim.x >> 5)) {
        const int64_t chunk = job / parts;
        const int first = int(chunk) * kStrip - kStrip, part = int(job - chunk * parts), hv0 = few ? part >> 1 : part * each;  // first: of a window of 48 tokens
        const auto slot_of = [&](int64_t i) -> int64_t {
            const int64_t slot = i >= 0 && i < a.n_new ? a.slots[i] : -1;
            return (slot >> shift) < kv.n_pages ? slot : -1;
        };
        const int64_t s0 = slot_of(int64_t(first) + lane), s1 = lane < kStrip ? slot_of(int64_t(first) + 32 + lane) : -1;
        // Tokens whose slot begins a strip that they and the 15 behind them fill; bit i: the window's token i.
        int64_t n0 = __shfl_down_sync(FULL, s0, 1);
        const int64_t n1 = __shfl_down_sync(FULL, s1, 1), s32 = __shfl_sync(FULL, s1, 0);
        if (lane == 31) n0 = s32;
        uint64_t run = __ballot_sync(FULL, s0 >= 0 && n0 == s0 + 1) | uint64_t(__ballot_sync(FULL, lane < kStrip - 1 && s1 >= 0 && n1 == s1 + 1)) << 32;
        run &= run >> 1;
        run &= run >> 2;
        run &= run >> 4;
        run &= run >> 7;  // 15 in a row
        const uint32_t fills = uint32_t(run) & __ballot_sync(FULL, s0 >= 0 && s0 % kStrip == 0);
        const uint32_t before = fills & 0xfffeu, here = fills >> 16;  // at most one each that reaches into the chunk
        const int done = few ? kStrip : before ? 32 - __clz(before) - 1 + kStrip : kStrip, own = !few && here ? __ffs(here) - 1 + kStrip : 2 * kStrip;
#pragma unroll 1
        for (int hw = 2 * hv0; hw < 2 * min(hv0 + each, 2 * H); ++hw) {  // the chunk's tokens that fill no strip; the strip that begins in it
            const int hv = hw >> 1, whole = hw & 1, v = hv >= H, h = hv - v * H;
            if (whole ? own == 2 * kStrip : done >= own) continue;
            const uint16_t *const source = static_cast<const uint16_t *>(v ? a.v : a.k) + h * (v ? a.vh : a.kh) + 8 * t;
            const int64_t stride = v ? a.vt : a.kt;
            unsigned char *const heads = static_cast<unsigned char *>(kv.pool) + ((int64_t(a.layer) * 2 + v) * H + h) * kv_head_bytes(kv);
            const auto strip_at = [&](int64_t slot) {
                return heads + (slot >> shift) * kv_page_bytes(kv) + int(slot & (P - 1)) / kStrip * kv_strip_bytes(kv);
            };
#pragma unroll 1
            for (int e = few ? part & 1 : 0; e < (few ? (part & 1) + 1 : 2); ++e) {
                const int at = (whole ? own : kStrip) + g + 8 * e;  // in the window
                const int64_t lo_slot = __shfl_sync(FULL, s0, at & 31), hi_slot = __shfl_sync(FULL, s1, at & 31), slot = at < 32 ? lo_slot : hi_slot;
                const bool in = whole || (at >= done && at < own && slot >= 0);
                const uint16_t *from = source + (int64_t(first) + at) * stride;
                uint4 x[DG];
#pragma unroll
                for (int j = 0; j < DG; ++j) {
                    x[j] = make_uint4(0, 0, 0, 0);
                    if (!in || 32 * j + 8 * t >= D) continue;
                    if (VEC) {
                        x[j] = __ldcs(reinterpret_cast<const uint4 *>(from + 32 * j));
                    } else {
                        const uint16_t *y = from + 32 * j;
                        x[j] = make_uint4(y[0] | uint32_t(y[1]) << 16, y[2] | uint32_t(y[3]) << 16, y[4] | uint32_t(y[5]) << 16, y[6] | uint32_t(y[7]) << 16);
                    }
                }
                // Each lane's lowest, and highest with its sign turned, so that the lower of both is taken at once; then those of group t.
                uint32_t ends[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    ends[j] = BF ? 0x7f807f80u : 0x7c007c00u;  // none: above all
                    if (j < DG && 32 * j + 8 * t < D) {
                        const uint4 y = x[j < DG ? j : 0];
                        const uint32_t least = min16<BF>(min16<BF>(y.x, y.y), min16<BF>(y.z, y.w)), most = max16<BF>(max16<BF>(y.x, y.y), max16<BF>(y.z, y.w)) ^ 0x80008000u;
                        ends[j] = min16<BF>(__byte_perm(least, most, 0x5410), __byte_perm(least, most, 0x7632));
                    }
                }
                const bool odd = t & 1, high = t & 2;
                const uint32_t l0 = min16<BF>(odd ? ends[1] : ends[0], __shfl_xor_sync(FULL, odd ? ends[0] : ends[1], 1));
                const uint32_t l1 = min16<BF>(odd ? ends[3] : ends[2], __shfl_xor_sync(FULL, odd ? ends[2] : ends[3], 1));
                const uint32_t mine = min16<BF>(high ? l1 : l0, __shfl_xor_sync(FULL, high ? l0 : l1, 2));
                const float low = wide<BF>(mine, 0), up = -wide<BF>(mine, 1);
                const bool finite = low * 0.f == 0.f && up * 0.f == 0.f;
                const uint32_t step = finite ? step_of<BF>(low, up) : 0x7fffu, scale = step | (finite ? mine << 16 : 0x7fff0000u);
                // One over the step, to the nearest float; 0 where that, or the quotients by the step, may leave the range, where the step
                // leaves more than 15.5 of them, and where there is none.
                const float of = wide<BF>(scale, 0);
                // (of 1 where it is not used: the call takes a longer way out of the range)
                const bool plain = of > (BF ? 0x1p-100f : 0x1p-18f) && of < (BF ? 0x1p100f : 0x1p14f);
                float over = __frcp_rn(plain ? of : 1.f);
                if (!plain) over = 0.f;
                // A difference that is not exact is one of numbers whose last places lie more than 24 powers of two under the first: one is
                // below 2^-15 (bfloat16) or 2^-12 (float16) of the difference.  It is rounded to a border only if the larger number lies
                // that near to one: in bfloat16 on it, as borders have 13 bits; in float16 (16 bits) within a 2^12th of -lo.  So where -lo
                // is not that near to one of the step's borders, and lo is 0 or not small, it does not matter.
                const float q0 = -low * over, q1 = fmaf(fmaf(-q0, of, -low), over, q0), apart = fabsf(q1 - (q1 + 0x1.8p23f - 0x1.8p23f));
                const bool on = BF ? apart == 0.5f : apart > 0.5f - 0x1p-8f, small = low != 0.f && fabsf(low) < up * (BF ? 0x1p-14f : 0x1p-10f);
                over = on || small ? -over : over;
                uint32_t code[DG];
                const auto quantise = [&](auto values, int j) {  // the codes' places in a word: those of values or of keys
                    constexpr bool V = decltype(values)::value;
                    const uint32_t sc = __shfl_sync(FULL, scale, j, 4);
                    const float in1 = __shfl_sync(FULL, over, j, 4), inv = fabsf(in1), s = wide<BF>(sc, 0), lo = wide<BF>(sc, 1);
                    const uint4 y = x[j];
                    // The difference, its quotient by the step to the nearest float (Markstein, IBM J. Res. Dev. 34, 1990: a product with the rounded
                    // reciprocal, corrected by its remainder, which is exact here as a step has 11 bits at most), and that to the nearest whole number,
                    // ties to even.  Where the difference is exact, a quotient on a border is a float; one next to it is more than half of a float's
                    // unit away, as the difference is a float too.
                    uint32_t w = 0u - 0x4b400000u * 0x11111111u;
                    const auto value = [&](int q) { return wide<BF>(q < 2 ? y.x : q < 4 ? y.y : q < 6 ? y.z : y.w, q % 2); };
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float d = value(q) - lo, q0 = d * inv, q1 = fmaf(fmaf(-q0, s, d), inv, q0);
                        w += __float_as_uint(q1 + 0x1.8p23f) << (V ? 4 * q : 4 * (q / 2) + 16 * (q % 2));
                    }
                    if (!(in1 > 0.f)) {
                        uint32_t cut = 0;  // differences that are not exact
                        if (in1 < 0.f) {
#pragma unroll
                            for (int q = 0; q < 8; ++q) cut |= __float_as_uint(__fsub_rz(value(q), lo)) ^ __float_as_uint(__fsub_ru(value(q), lo));
                        }
                        if (cut || in1 == 0.f) w = s > 0.f && 32 * j + 8 * t < D ? codes_exactly<BF>(y, lo, s, V) : 0;
                    }
                    code[j] = w;
                };
                if (v) {
#pragma unroll
                    for (int j = 0; j < DG; ++j) quantise(std::true_type(), j);
                } else {
#pragma unroll
                    for (int j = 0; j < DG; ++j) quantise(std::false_type(), j);
                }
                const auto store = [&](unsigned char *to, int T) {
                    if (v == 0) {
                        uint32_t *const c = reinterpret_cast<uint32_t *>(to + 16 * DG * T + 4 * DG * t), *const sc = reinterpret_cast<uint32_t *>(to + 256 * DG + 4 * DG * T);
                        if constexpr (DG == 4) *reinterpret_cast<uint4 *>(c) = make_uint4(code[0], code[1], code[2], code[3]);
#pragma unroll
                        for (int j = 0; j < DG && DG != 4; ++j) c[j] = code[j];
                        if (t < DG) sc[t] = scale;
                    } else {
                        unsigned char *const c = to + 128 * DG * (T / 8) + 4 * DG * (8 * t + T % 8 / 2) + 2 * (T % 2);
                        uint16_t *const sc = reinterpret_cast<uint16_t *>(to + 256 * DG + 8 * DG * (T / 2) + 2 * (T % 2) + 8 * t);
#pragma unroll
                        for (int j = 0; j < DG; ++j) {
                            *reinterpret_cast<uint16_t *>(c + 4 * j) = uint16_t(code[j]);
                            *reinterpret_cast<uint16_t *>(c + 16 * DG + 4 * j) = uint16_t(code[j] >> 16);
                        }
                        if (t < DG) {
                            sc[0] = uint16_t(scale);
                            sc[2] = uint16_t(scale >> 16);
                        }
                    }
                };
                if (whole) store(image, g + 8 * e);
                else if (in) store(strip_at(slot), int(slot & (kStrip - 1)));
            }
            if (whole) {
                __syncwarp();
                uint4 *const to = reinterpret_cast<uint4 *>(strip_at(__shfl_sync(FULL, s0, own)));
#pragma unroll
                for (int i = 0; i < (20 * DG + 31) / 32; ++i)
                    if (lane + 32 * i < 20 * DG) __stcs(to + lane + 32 * i, reinterpret_cast<const uint4 *>(image)[lane + 32 * i]);
                __syncwarp();
            }
        }
    }
}

// ---- reading ---------------------------------------------------------------------------------------------------

// Entry i's rows lie on strips of its sequence; they have the numbers from cu[i] / 16 + 2 i on, which leave each entry at least as many
// as it needs.
__device__ __forceinline__ int64_t first_strip(const int32_t *cu, int i) { return cu[i] / kStrip + 2 * int64_t(i); }

// The last entry whose strips begin at or before x, by a warp: a 32nd of what is left at a time.
__device__ __forceinline__ int entry_of_strip(const int32_t *cu, int n, int64_t x) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n;  // in [lo, hi)
    while (hi - lo > 1) {
        const int each = (hi - lo + 31) / 32, at = lo + lane * each;
        const int k = __popc(__ballot_sync(FULL, at < hi && first_strip(cu, at) <= x));
        lo += max(k - 1, 0) * each;
        hi = min(lo + each, hi);
    }
    return lo;
}

// A warp for each strip and kv head, keys and values: all loads before the first store.
template <int DG, bool BF>
__global__ void __launch_bounds__(kRead) k_read(const sim_kv kv, const KvRead r) {
    kv_wait_previous();
    const int lane = threadIdx.x & 31, H = kv.n_kv_heads, D = kv.head_dim, P = kv.page_size;
    // Offsets of a few entries are searched where they have been read to, in shared memory.
    __shared__ int32_t few_cu[kFewEntries + 1];
    const bool few = r.n <= kFewEntries;
    const int32_t *const cu = few ? few_cu : r.cu;
    bool order = true;
    for (int i = threadIdx.x; i < r.n; i += kRead) {
        const int a = r.cu[i], b = r.cu[i + 1];
        order = order && 0 <= a && a <= b && b <= r.total;
        if (few) few_cu[i] = a;
        if (few && i + 1 == r.n) few_cu[i + 1] = b;
    }
    order = __syncthreads_and(order);
    if (!order && blockIdx.x == 0 && threadIdx.x == 0) atomicMin(kv.status, SIM_E_INVAL);
    uint16_t *const to[2] = {static_cast<uint16_t *>(r.k), static_cast<uint16_t *>(r.v)};
    const auto row = [&](int v, int y, int h) { return to[v] + y * (v ? r.vt : r.kt) + h * (v ? r.vh : r.kh); };
    const auto zeros = [&](int y, int h) {
        for (int d = 8 * lane; d < 2 * D; d += 256) *reinterpret_cast<uint4 *>(row(d >= D, y, h) + (d >= D ? d - D : d)) = make_uint4(0, 0, 0, 0);
    };
    const int64_t warp0 = int64_t(blockIdx.x) * (kRead / 32) + (threadIdx.x >> 5), warps = int64_t(gridDim.x) * (kRead / 32);
    const int64_t x0 = order && r.n > 0 ? first_strip(cu, 0) : 0, all = order && r.n > 0 ? (first_strip(cu, r.n) - x0) * H : 0;
    for (int64_t z = warp0; z < all; z += warps) {
        const int64_t x = x0 + z / H;
        const int h = int(z % H), i = entry_of_strip(cu, r.n, x), a = cu[i], count = cu[i + 1] - a, nth = int(x - first_strip(cu, i));
        if (count == 0) continue;
        const int s = r.seqs[i], f = r.first ? r.first[i] : 0;
        const bool known = unsigned(s) < unsigned(kv.max_seqs) && f >= 0 && int64_t(f) + count <= int64_t(kv.max_pages) * P;
        const int T0 = known ? (f / kStrip + nth) * kStrip : 0;  // token of the strip's first place
        // the length and the page at once: a strip past the entry's tokens may have none
        const int length = known ? kv.length[s] : 0, page = known && T0 < f + count ? kv.table[int64_t(s) * kv.max_pages + T0 / P] : -1;
        if (!known || f + count > length) {
            if (lane == 0) atomicMin(kv.status, SIM_E_INVAL);
            for (int y = nth * kStrip; y < min(nth * kStrip + kStrip, count); ++y) zeros(a + y, h);
            continue;
        }
        if (T0 >= f + count) continue;
        const int y0 = a - f + T0;
        const bool there = unsigned(page) < unsigned(kv.n_pages);
        const auto in = [&](int T) { return T0 + T >= f && T0 + T < f + count; };
        const unsigned char *const base = static_cast<const unsigned char *>(kv.pool) + (there ? page : 0) * kv_page_bytes(kv) +
                                          (int64_t(r.layer) * 2 * H + h) * kv_head_bytes(kv);
        if (!there) {
            for (int T = 0; T < kStrip; ++T)
                if (in(T)) zeros(y0 + T, h);
            continue;
        }
        if constexpr (DG == 0) {  // 16-bit floats
            const int vec = D / 8;
            uint4 keep[2][8];  // 16 tokens of 16 times 16 bytes at most
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = lane + 32 * e, T = at / vec;
                    if (at < kStrip * vec && in(T))
                        keep[v][e] = __ldcs(reinterpret_cast<const uint4 *>(base + v * (int64_t(H) * kv_head_bytes(kv)) + (T0 % P) * (2 * D)) + at);
                }
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = lane + 32 * e, T = at / vec;
                    if (at < kStrip * vec && in(T)) __stcs(reinterpret_cast<uint4 *>(row(v, y0 + T, h)) + at % vec, keep[v][e]);
                }
        } else {
            const int g = lane >> 2, t = lane & 3;
            const unsigned char *const ks = base + (T0 % P) / kStrip * (320 * DG), *const vs = ks + H * kv_head_bytes(kv);
            uint32_t kc[2][DG], kq[2][DG], vc[2][DG], vq[2][2 * DG];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                words<DG>(ks + 16 * DG * (g + 8 * e) + 4 * DG * t, kc[e]);
                words<DG>(ks + 256 * DG + 4 * DG * (g + 8 * e), kq[e]);
                words<DG>(vs + 128 * DG * e + 4 * DG * lane, vc[e]);
                words<2 * DG>(vs + 256 * DG + 8 * DG * (t + 4 * e), vq[e]);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int T = g + 8 * e;
                if (!in(T)) continue;
                uint16_t *const o = row(0, y0 + T, h) + 8 * t;
#pragma unroll
                for (int j = 0; j < DG; ++j) {
                    uint32_t x4[4];
                    values4<BF>(kc[e][j], low_twice(kq[e][j]), high_twice(kq[e][j]), x4);
                    if (32 * j + 8 * t < D) __stcs(reinterpret_cast<uint4 *>(o + 32 * j), make_uint4(x4[0], x4[1], x4[2], x4[3]));
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int T = 8 * e + 2 * t;
                uint16_t *const o = row(1, y0 + T, h) + 4 * g;
#pragma unroll
                for (int j = 0; j < DG; ++j) {
                    uint32_t x4[4];
                    values4<BF>(vc[e][j], vq[e][2 * j], vq[e][2 * j + 1], x4);
                    if (32 * j + 4 * g >= D) continue;
                    if (in(T)) __stcs(reinterpret_cast<uint2 *>(o + 32 * j), make_uint2(__byte_perm(x4[0], x4[1], 0x5410), __byte_perm(x4[2], x4[3], 0x5410)));
                    if (in(T + 1)) __stcs(reinterpret_cast<uint2 *>(o + r.vt + 32 * j), make_uint2(__byte_perm(x4[0], x4[1], 0x7632), __byte_perm(x4[2], x4[3], 0x7632)));
                }
            }
        }
    }
    // rows of no entry
    const int before = order && r.n > 0 ? cu[0] : r.total, after = order && r.n > 0 ? cu[r.n] : r.total;
    const int64_t rest = (int64_t(before) + r.total - after) * H;
    for (int64_t z = warp0; z < rest; z += warps) {
        const int y = int(z / H);
        zeros(y < before ? y : y - before + after, int(z % H));
    }
}

int blocks_for(int64_t items, int per_block, int per_sm) {
    return int(std::min<int64_t>(std::max<int64_t>(1, (items + per_block - 1) / per_block), int64_t(kv_sm_count()) * per_sm));
}

}  // namespace

cudaError_t launch_kv_write_4bit(const sim_kv &kv, const KvWrite &w, cudaStream_t st) {
    const auto aligned = [](const void *p, int64_t a, int64_t b) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && a % 8 == 0 && b % 8 == 0; };
    const bool vec = aligned(w.k, w.kt, w.kh) && aligned(w.v, w.vt, w.vh);
    using Fn = void (*)(const sim_kv, const KvWrite, int, int);
    constexpr Fn of[2][2][4] = {{{k_write_4bit<1, false, false>, k_write_4bit<2, false, false>, k_write_4bit<3, false, false>, k_write_4bit<4, false, false>},
                                 {k_write_4bit<1, false, true>, k_write_4bit<2, false, true>, k_write_4bit<3, false, true>, k_write_4bit<4, false, true>}},
                                {{k_write_4bit<1, true, false>, k_write_4bit<2, true, false>, k_write_4bit<3, true, false>, k_write_4bit<4, true, false>},
                                 {k_write_4bit<1, true, true>, k_write_4bit<2, true, true>, k_write_4bit<3, true, true>, k_write_4bit<4, true, true>}}};
    const int64_t chunks = (int64_t(w.n_new) + kStrip - 1) / kStrip;
    const int64_t heads = chunks * 2 * kv.n_kv_heads;
    // Heads that a warp takes, so that what it learns of the slots serves all, as long as there are warps enough for that.  k_write_4bit by
    // per_sm, with 1, 2, 4 heads (8 heads of 128, bfloat16 | 3 heads of 80, float16), us: 48: 23, 25, 36 | 21, 23, 33; 140: 44, 46, 54 | 40, 42,
    // 52; 284: 76, 74, 81 | 68, 66, 79; 400: 103, 99, 103 | 93, 89, 101; 700: 171, 158, 160 | 154, 142, 156; 1700: 400, 359, 351 | 359, 324, 343.
    // So 2 is right from some 200 on, where 96 takes it (2 us too many in between), and 4 from some 800 on if it divides the heads: with
    // 6 heads of keys and values, every second warp has half of them, and it costs 6 to 13 %.
    const int64_t per_sm = heads / kv_sm_count();
    const int few = per_sm < 4, each = per_sm < 96 ? 1 : per_sm < 512 ? 2 : 4, threads = few ? 64 : kWrite;
    const int blocks = blocks_for(few ? 2 * heads : chunks * ((2 * kv.n_kv_heads + each - 1) / each), threads / 32, 4096);
    return launch_chained(of[kv_bf(kv)][vec][kv_dim_groups(kv) - 1], blocks, threads, 0, st, kv, w, each, few);
}

cudaError_t launch_kv_read(const sim_kv &kv, const KvRead &r, cudaStream_t st) {
    const int G = kv_4bit(kv) ? kv_dim_groups(kv) : 0;
    using Fn = void (*)(const sim_kv, const KvRead);
    constexpr Fn of[2][5] = {{k_read<0, false>, k_read<1, false>, k_read<2, false>, k_read<3, false>, k_read<4, false>},
                             {k_read<0, false>, k_read<1, true>, k_read<2, true>, k_read<3, true>, k_read<4, true>}};
    const int blocks = blocks_for((int64_t(r.total) / kStrip + 2 * int64_t(r.n) + 1) * kv.n_kv_heads, kRead / 32, 64);
    return launch_chained(of[kv_bf(kv)][G], blocks, kRead, 0, st, kv, r);
}

}  // namespace simgb
