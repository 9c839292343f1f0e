// Keys and values of a 4-bit cache: quantised as they are written, and read back (16-bit caches are read here too).
#include <algorithm>
#include <climits>

#include "sim.h"
#include "sim_kv_4bit.cuh"

namespace simgb {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int kWrite = 256, kRead = 256;  // threads

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
        if (large) step += 3 << 7;
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

// A lane has 8 of a group's values at columns 8 u and 8 more at 16 + 8 u, the other half of them is its neighbour's.
// VEC: the sources are 16-byte aligned.
template <bool BF, bool VEC>
__global__ void __launch_bounds__(kWrite) k_write_4bit(const sim_kv kv, const KvWrite a, const FastDiv per_row, const FastDiv groups) {
    kv_wait_previous();
    const int P = kv.page_size, D = kv.head_dim, G = int(groups.d), H = kv.n_kv_heads, shift = __ffs(P) - 1;
    const int64_t all = int64_t(a.n_new) * 2 * per_row.d;
    for (int64_t i0 = int64_t(blockIdx.x) * kWrite; i0 < all; i0 += int64_t(gridDim.x) * kWrite) {
        const int64_t i = min(i0 + threadIdx.x, all - 1);  // lanes past the end (of all, an even number) make the last one's pair again, or its neighbour's
        int row, r;
        if (all <= INT_MAX) {
            row = int(per_row.div(uint32_t(i)));
            r = int(i - int64_t(row) * per_row.d);
        } else {
            row = int(i / per_row.d);
            r = int(i % per_row.d);
        }
        const int tok = row >> 1, v = row & 1, u = r & 1, h = int(groups.div(uint32_t(r >> 1))), j = (r >> 1) - h * G;
        const int64_t slot = a.slots[tok], page = slot >> shift;
        const bool there = slot >= 0 && page < kv.n_pages && i0 + threadIdx.x < all;
        const uint16_t *const from = static_cast<const uint16_t *>(v ? a.v : a.k) + tok * (v ? a.vt : a.kt) + h * (v ? a.vh : a.kh) + 32 * j + 8 * u;
        const int left = D - 32 * j - 8 * u;  // columns from the first of this lane's on
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (16 * e >= left) {  // none: as others of the group, so that neither lowest nor highest is changed
                x[4 * e] = x[4 * e + 1] = x[4 * e + 2] = x[4 * e + 3] = e > 0 ? x[0] : 0;
            } else if (VEC) {
                const uint4 y = __ldcs(reinterpret_cast<const uint4 *>(from + 16 * e));
                x[4 * e] = y.x, x[4 * e + 1] = y.y, x[4 * e + 2] = y.z, x[4 * e + 3] = y.w;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) x[4 * e + q] = from[16 * e + 2 * q] | uint32_t(from[16 * e + 2 * q + 1]) << 16;
            }
        }
        uint32_t least = x[0], most = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) {
            least = min16<BF>(least, x[e]);
            most = max16<BF>(most, x[e]);
        }
        least = min16<BF>(least, least >> 16 | least << 16);
        most = max16<BF>(most, most >> 16 | most << 16);
        const uint32_t mine = __byte_perm(least, most, 0x5410), other = __shfl_xor_sync(FULL, mine, 1);
        const bool both = D - 32 * j > 8;  // the group has columns for the second lane
        least = both ? min16<BF>(mine, other) & 0xffffu : (u ? other : mine) & 0xffffu;
        most = both ? max16<BF>(mine, other) >> 16 : (u ? other : mine) >> 16;
        float lo = wide16<BF>(least);
        const float hi = wide16<BF>(most);
        const bool finite = lo * 0.f == 0.f && hi * 0.f == 0.f;
        const uint32_t step = finite ? step_of<BF>(lo, hi) : 0x7fffu, base = finite ? least : 0x7fffu;
        float s = finite ? wide16<BF>(step) : 0.f;
        // Tiny steps, whose reciprocals overflow, and large ones, whose differences do, after a multiplication by a power of two.
        const float more = BF && s > 0.f && s < 0x1p-60f ? 0x1p60f : BF && s > 0x1p110f ? 0x1p-8f : 1.f;
        s *= more;
        lo = finite ? lo * more : 0.f;
        float inv = 0.f;
        if (s > 0.f) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));  // f16's least is 2^-24
        uint32_t w[4];  // of columns 2 q and 2 q + 1 at bits 4 q of two halves, for 8 columns; or of four and four
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float part[2] = {0.f, 0.f};  // four codes each, below 2^16: exact
            constexpr float kScale[4] = {1.f, 16.f, 256.f, 4096.f};
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float val = wide<BF>(x[4 * e + q / 2], q % 2), t = fmaf(val, more, -lo), near = fmaf(t, inv, 0x1.8p23f) - 0x1.8p23f;
                float code = near;  // the quotient, within 2^-18 where it is below 16, to the nearest
                if (fabsf(fmaf(t, inv, -near)) > 0.5f - 0x1p-17f) code = code_at_border(val * more, lo, t, t * inv, s);
                code = fminf(code, 15.f);
                part[v ? q / 4 : q % 2] = fmaf(code, kScale[v ? q % 4 : q / 2], part[v ? q / 4 : q % 2]);
            }
            w[2 * e] = finite ? uint32_t(part[0]) : 0;
            w[2 * e + 1] = finite ? uint32_t(part[1]) : 0;
        }
        if (!there) continue;
        unsigned char *const strip = static_cast<unsigned char *>(kv.pool) + page * kv_page_bytes(kv) +
                                     ((int64_t(a.layer) * 2 + v) * H + h) * kv_head_bytes(kv) + int(slot & (P - 1)) / kStrip * kv_strip_bytes(kv);
        const int T = int(slot & (kStrip - 1));
        if (v == 0) {
            uint32_t *const to = reinterpret_cast<uint32_t *>(strip + 16 * G * T + 4 * G * u + 4 * j);
            to[0] = w[0] | w[1] << 16;
            to[2 * G] = w[2] | w[3] << 16;
            if (u == 0) *reinterpret_cast<uint32_t *>(strip + 256 * G + 4 * G * T + 4 * j) = step | base << 16;
        } else {
            uint16_t *const to = reinterpret_cast<uint16_t *>(strip + 128 * G * (T / 8) + 4 * G * (T % 8 / 2) + 32 * G * u + 4 * j + 2 * (T % 2));
            to[0] = uint16_t(w[0]);
            to[8 * G] = uint16_t(w[1]);
            to[32 * G] = uint16_t(w[2]);
            to[40 * G] = uint16_t(w[3]);
            uint16_t *const sc = reinterpret_cast<uint16_t *>(strip + 256 * G + 8 * G * (T / 2) + 8 * j + 2 * (T % 2));
            sc[2 * u] = uint16_t(u ? base : step);
        }
    }
}

// ---- reading ---------------------------------------------------------------------------------------------------

// Entry i's rows lie on strips of its sequence; they have the numbers from cu[i] / 16 + 2 i on, which leave each entry at least as many
// as it needs.
__device__ __forceinline__ int64_t first_strip(const KvRead &r, int i) { return r.cu[i] / kStrip + 2 * int64_t(i); }

// The last entry whose strips begin at or before x, by a warp: a 32nd of what is left at a time.
__device__ __forceinline__ int entry_of_strip(const KvRead &r, int64_t x) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = r.n;  // in [lo, hi)
    while (hi - lo > 1) {
        const int each = (hi - lo + 31) / 32, at = lo + lane * each;
        const int k = __popc(__ballot_sync(FULL, at < hi && first_strip(r, at) <= x));
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
    bool order = true;
    for (int i = threadIdx.x; i < r.n; i += kRead) order = order && 0 <= r.cu[i] && r.cu[i] <= r.cu[i + 1] && r.cu[i + 1] <= r.total;
    order = __syncthreads_and(order);
    if (!order && blockIdx.x == 0 && threadIdx.x == 0) atomicMin(kv.status, SIM_E_INVAL);
    uint16_t *const to[2] = {static_cast<uint16_t *>(r.k), static_cast<uint16_t *>(r.v)};
    const auto row = [&](int v, int y, int h) { return to[v] + y * (v ? r.vt : r.kt) + h * (v ? r.vh : r.kh); };
    const auto zeros = [&](int y, int h) {
        for (int d = 8 * lane; d < 2 * D; d += 256) *reinterpret_cast<uint4 *>(row(d >= D, y, h) + (d >= D ? d - D : d)) = make_uint4(0, 0, 0, 0);
    };
    const int64_t warp0 = int64_t(blockIdx.x) * (kRead / 32) + (threadIdx.x >> 5), warps = int64_t(gridDim.x) * (kRead / 32);
    const int64_t x0 = order && r.n > 0 ? first_strip(r, 0) : 0, all = order && r.n > 0 ? (first_strip(r, r.n) - x0) * H : 0;
    for (int64_t z = warp0; z < all; z += warps) {
        const int64_t x = x0 + z / H;
        const int h = int(z % H), i = entry_of_strip(r, x), a = r.cu[i], count = r.cu[i + 1] - a, nth = int(x - first_strip(r, i));
        if (count == 0) continue;
        const int s = r.seqs[i], f = r.first ? r.first[i] : 0;
        if (unsigned(s) >= unsigned(kv.max_seqs) || f < 0 || int64_t(f) + count > kv.length[s] || kv.length[s] > kv.max_pages * P) {
            if (lane == 0) atomicMin(kv.status, SIM_E_INVAL);
            for (int y = nth * kStrip; y < min(nth * kStrip + kStrip, count); ++y) zeros(a + y, h);
            continue;
        }
        const int T0 = (f / kStrip + nth) * kStrip;  // token of the strip's first place
        if (T0 >= f + count) continue;
        const int page = kv.table[int64_t(s) * kv.max_pages + T0 / P], y0 = a - f + T0;
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
    const int before = order && r.n > 0 ? r.cu[0] : r.total, after = order && r.n > 0 ? r.cu[r.n] : r.total;
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
    const auto k = kv_bf(kv) ? (vec ? k_write_4bit<true, true> : k_write_4bit<true, false>) : vec ? k_write_4bit<false, true> : k_write_4bit<false, false>;
    const int G = kv_dim_groups(kv), per_row = 2 * G * kv.n_kv_heads;  // lanes for a token's keys, or its values
    const int blocks = blocks_for(int64_t(w.n_new) * 2 * per_row, kWrite, 4096);
    return launch_chained(k, blocks, kWrite, 0, st, kv, w, FastDiv(per_row), FastDiv(G));
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
