// Declarations shared by the C ABI of the paged cache (sim_kv_api.cpp) and its kernels (sim_kv.cu, sim_kv_attend.cu,
// sim_kv_heavy.cu, sim_kv_light.cu; of 4-bit caches sim_kv_4bit.cu, sim_kv_4bit_light.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "sim_kv.h"

namespace simgb {

constexpr int kKvMaxSeqs = 1 << 17;

// kv->scratch, in ints: a header, then per entry of a call its first new page, their number and its length before,
// then lists of pages (as many as the pool has): copies' sources and destinations, free pages.
constexpr int kKvHdr = 64;  // [0]: copies to make
__host__ __device__ inline int64_t kv_scratch_ints(const sim_kv &kv) { return kKvHdr + 3 * int64_t(kv.max_seqs) + 3 * int64_t(kv.n_pages); }
struct KvScratch {
    int32_t *hdr, *base, *need, *len, *src, *dst, *free;
};
__host__ __device__ inline KvScratch kv_scratch(const sim_kv &kv) {
    KvScratch s;
    s.hdr = static_cast<int32_t *>(kv.scratch);
    s.base = s.hdr + kKvHdr;
    s.need = s.base + kv.max_seqs;
    s.len = s.need + kv.max_seqs;
    s.src = s.len + kv.max_seqs;
    s.dst = s.src + kv.n_pages;
    s.free = s.dst + kv.n_pages;
    return s;
}

__host__ __device__ inline bool kv_bf(const sim_kv &kv) { return kv.dtype == SIM_KV_BF16 || kv.dtype == SIM_KV_BF16_4BIT; }
__host__ __device__ inline bool kv_4bit(const sim_kv &kv) { return kv.dtype == SIM_KV_BF16_4BIT || kv.dtype == SIM_KV_F16_4BIT; }
// A 4-bit cache: groups of 32 values of a token's head, the last one shorter; strips of 16 tokens of a head, 20 bytes a token and group.
constexpr int kStrip = 16;
__host__ __device__ inline int kv_dim_groups(const sim_kv &kv) { return (kv.head_dim + 31) / 32; }
__host__ __device__ inline int64_t kv_strip_bytes(const sim_kv &kv) { return 20 * kStrip * kv_dim_groups(kv); }
__host__ __device__ inline int64_t kv_layer_elems(const sim_kv &kv) { return 2 * int64_t(kv.n_kv_heads) * kv.page_size * kv.head_dim; }  // 16-bit caches
__host__ __device__ inline int64_t kv_head_bytes(const sim_kv &kv) {  // a page's keys, or values, of one head
    return kv.page_size * (kv_4bit(kv) ? 20 * int64_t(kv_dim_groups(kv)) : 2 * int64_t(kv.head_dim));
}
__host__ __device__ inline int64_t kv_page_bytes(const sim_kv &kv) { return kv.n_layers * (2 * int64_t(kv.n_kv_heads)) * kv_head_bytes(kv); }

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 by a multiplication: with 2^(k-1) < d <= 2^k, m = ceil(2^(31+k) / d)
// < 2^32 gives floor(n m / 2^(31+k)), since n (m d - 2^(31+k)) < n 2^k <= 2^(31+k).
struct FastDiv {
    uint32_t d, m, s;
    __host__ __device__ FastDiv() : d(1), m(0), s(0) {}
    __host__ explicit FastDiv(uint32_t dd) : d(dd), m(0), s(0) {
        if (dd > 1) {
            uint32_t k = 1;
            while ((uint64_t(1) << k) < dd) ++k;
            m = uint32_t(((uint64_t(1) << (31 + k)) + dd - 1) / dd);
            s = k - 1;
        }
    }
#ifdef __CUDACC__
    __device__ uint32_t div(uint32_t n) const { return d == 1 ? n : __umulhi(n, m) >> s; }
#endif
};

cudaError_t launch_kv_extend(const sim_kv &kv, int32_t n, const int32_t *seqs, const int32_t *cu_new, int32_t n_new,
                             int64_t *slots, cudaStream_t st);
cudaError_t launch_kv_copy(const sim_kv &kv, int32_t n, const int32_t *src, const int32_t *dst, cudaStream_t st);
cudaError_t launch_kv_fork(const sim_kv &kv, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *tokens,
                           cudaStream_t st);
cudaError_t launch_kv_free(const sim_kv &kv, int32_t n, const int32_t *seqs, const int32_t *keep, cudaStream_t st);
cudaError_t launch_kv_compact(const sim_kv &kv, int32_t *to, cudaStream_t st);
struct KvWrite {
    const void *k, *v;
    int64_t kt, kh, vt, vh;  // strides in elements
    const int64_t *slots;
    int32_t layer, n_new;
};
cudaError_t launch_kv_write(const sim_kv &kv, const KvWrite &w, cudaStream_t st);

struct KvRead {
    const int32_t *seqs, *cu, *first;
    void *k, *v;
    int64_t kt, kh, vt, vh;  // strides in elements
    int32_t layer, n, total;
};
cudaError_t launch_kv_read(const sim_kv &kv, const KvRead &r, cudaStream_t st);
cudaError_t launch_kv_write_4bit(const sim_kv &kv, const KvWrite &w, cudaStream_t st);

// Items of more than 32 rows are heavy, the others light: two lists, each divided among blocks of its own.
constexpr int kAttRows = 256;   // query rows of a heavy item, at most
constexpr int kLightRows = 32;  // of a light one
__host__ __device__ constexpr int kv_rows(int light) { return light ? kLightRows : kAttRows; }
// Batches that look like single tokens (no more of them than entries, no groups): all rows are light items, as many as it takes
// if an entry has many after all, and the heavy kernel is not launched: over an empty list it costs the
// host 1.6 us and the GPU 2 to 3 us of a step that takes 26.
__host__ __device__ inline bool kv_light_only(const sim_kv &kv, const sim_kv_batch &b) {
    const int64_t G = b.q_heads / kv.n_kv_heads;
    return b.n_q * G <= kLightRows || (b.n_groups == 0 && G <= kLightRows && b.n_q <= b.n);
}
// Rows of a light item, at most.  Of a 4-bit cache, by what entries have on average: more than 16 do not leave enough registers (when chosen: 128
// sequences of up to 2000 keys: with 16 query heads for each of 8 kv heads 75 us with 16 rows, 96 us with 8, 122 us with 32 at a time; with 32
// heads for each of 4 85, 113, 89 us; with 1 to 4 tokens of 8 heads 135, 179, 150 us).
// Every kernel asks for it, so there is no division (a 64-bit one for each kernel of a call takes 2 us).
__host__ __device__ inline int kv_light_shift(const sim_kv &kv, const sim_kv_batch &b) {  // its logarithm
    const int64_t rows = int64_t(b.n_q) * (b.q_heads / kv.n_kv_heads);
    return !kv_4bit(kv) ? 5 : rows <= 8 * int64_t(b.n > 0 ? b.n : 1) ? 3 : 4;
}
__host__ __device__ inline int kv_light_rows(const sim_kv &kv, const sim_kv_batch &b) { return 1 << kv_light_shift(kv, b); }
static_assert(kLightRows == 1 << 5, "kv_light_shift");
// Blocks of the light list on an SM: three of a 4-bit cache where 8 rows a pass leave enough registers (384 sequences of up to 2600 keys, when
// chosen: 167 instead of 183 us with two).
__host__ __device__ inline int kv_per_sm(const sim_kv &kv, const sim_kv_batch &b) { return kv_light_rows(kv, b) == 8 ? 3 : 2; }
constexpr int kTileKeys = 128;  // keys of a tile
// What taking up an item and writing its results costs, in tiles: on the line of work, that much lies before an item's
// tiles.  (4-bit caches, 384 sequences of up to 2600 keys, when chosen: 185, 183, 188, 193 us with 1, 2, 3, 4.)
__host__ __device__ inline int kv_lead(const sim_kv &kv, int light) { return light ? (kv_4bit(kv) ? 2 : 1) : 4; }
__host__ __device__ inline int kv_span(int tiles, int lead) { return tiles > 0 ? tiles + lead : 0; }

// A run of query rows (token x head of the group, for every kv head alike) against a range of one table's keys.
struct alignas(16) KvItem {
    int32_t q0;       // query token of row 0 of its source
    int32_t row0;     // first row within the source
    int32_t rows;     // 1 .. kv_rows
    int32_t seq;      // row of the table
    int32_t kv0, kv1; // keys
    int32_t pos0;     // position of token q0: token q0 + t sees the keys up to pos0 + t
    int32_t tiles;
    int64_t unit;     // spans of the items before, all kv heads
    int64_t row_off;  // rows of the items before, all kv heads
    int32_t partial;  // its rows have another item too: always through the workspace
    int32_t pad[3];
};
static_assert(sizeof(KvItem) == 64, "KvItem");

// Where the rows of items come from: a group's prefix, or an entry's own keys.  Groups come first, then entries.
struct alignas(16) KvSource {
    int32_t q0, rows;         // first query token, rows of a kv head
    int32_t seq, kv0, kv1;    // row of the table, keys
    int32_t pos0;             // as KvItem's
    int32_t heavy0, n_heavy;  // its heavy items
    int32_t light0;           // the first of its light items, after them: one, in a 4-bit cache and with kv_light_only perhaps more
    int32_t prefix;           // source of the prefix that it shares, or -1
    int32_t blind;            // some of its rows see no key
    int32_t tiles;            // of its first light item, whose .unit and .row_off follow
    int64_t unit, row_off;
};
static_assert(sizeof(KvSource) == 64, "KvSource");

// A place where the stretches of two blocks meet within an item that has no prefix, the item's first: k_combine joins
// its pieces there.
struct alignas(16) KvCut {
    int64_t row;        // partial results of the first piece
    int32_t n, pad;     // pieces
    int32_t q0, row0, rows, h;
};
static_assert(sizeof(KvCut) == 32, "KvCut");

// b->plan: header, where each block's stretch begins and what it cuts, the sources and the pages that entries share
// with their group's first, the items; numbers for searches: each source's first items, pages used by groups.
constexpr int kKvMaxSms = 256;
struct KvPlan {
    int32_t *hdr;       // heavy, and 16 further light: [0] items, [2..3] spans in all, [4..5] of each block, [6] left over,
                        // [7] cuts, [10] lead; [1] offsets in order, [17] entries to join, [24..25] rows of the heavy items
    KvCut *cut[2];      // as many as there are, in any order
    KvSource *source;   // [n_groups + n]
    KvItem *items[2];
    int32_t *start[2];  // [kv_blocks] item in which each block's stretch begins
    int32_t *first[2];  // [n_groups + n + 1]
    int32_t *used;      // [n_groups]
    int32_t *alone;     // [n_groups]
    int32_t *same;      // [n]
    int32_t *join;      // [n] entries with a shared prefix or rows without keys, in any order
    int64_t bytes;
    int32_t max_heavy;
    int64_t max_light;
};
__host__ __device__ inline KvPlan kv_plan(const sim_kv &kv, const sim_kv_batch &b) {
    KvPlan p;
    const int64_t G = b.q_heads / kv.n_kv_heads, src = int64_t(b.n_groups) + b.n;
    // each query row is in one group and one entry; a source has one item of fewer than kAttRows rows at most
    const int64_t whole = 2 * (int64_t(b.n_q) * G / kAttRows) + src, small = 2 * (int64_t(b.n_q) * G / (kLightRows + 1));
    p.max_heavy = int32_t((whole < small ? whole : small) + 1);
    // light items: where heavy ones take the most rows, those of 32 rows a source at most, or of all rows, each in an entry and perhaps in a group
    const int shift = kv_light_shift(kv, b);
    const int64_t most = src << (5 - shift), many = src + ((int64_t(b.n_q) * G << (b.n_groups > 0)) >> shift);
    p.max_light = !kv_light_only(kv, b) && most < many ? most : many;
    p.hdr = static_cast<int32_t *>(b.plan);
    p.cut[0] = reinterpret_cast<KvCut *>(p.hdr + 32);
    p.cut[1] = p.cut[0] + kKvMaxSms;
    p.source = reinterpret_cast<KvSource *>(p.cut[1] + 3 * kKvMaxSms);
    p.items[0] = reinterpret_cast<KvItem *>(p.source + src);
    p.items[1] = p.items[0] + p.max_heavy;
    p.start[0] = reinterpret_cast<int32_t *>(p.items[1] + p.max_light);
    p.start[1] = p.start[0] + kKvMaxSms;
    p.first[0] = p.start[1] + 3 * kKvMaxSms;
    p.first[1] = p.first[0] + src + 1;
    p.used = p.first[1] + src + 1;
    p.alone = p.used + b.n_groups;
    p.same = p.alone + b.n_groups;
    p.join = p.same + b.n;
    p.bytes = reinterpret_cast<char *>(p.join + b.n) - static_cast<char *>(b.plan);
    return p;
}
// Blocks of the two lists for a number of SMs.
__host__ __device__ inline int kv_blocks(int sms, int light, int per_sm = 2) { return light ? per_sm * sms : sms; }
// Partial results: rows of head_dim floats, then a float per row (log2 of the sum of exponentials).  A piece of an
// item begins at the rows before it plus room for the pieces that blocks have cut off before.
__host__ __device__ inline int64_t kv_partial_rows(const sim_kv &kv, const sim_kv_batch &b, int sms) {
    return 2 * int64_t(b.n_q) * b.q_heads + int64_t(kAttRows) * kv_blocks(sms, 0) + int64_t(kLightRows) * kv_blocks(sms, 1, kv_per_sm(kv, b));
}

struct KvAttend {
    const void *q;
    void *out;
    float *lse;
    float *part, *part_lse;
    int64_t qt, qh, ot, oh;  // strides in elements
    float scale_log2;
    int32_t layer;
    int32_t q_vec;           // q may be read 16 bytes at a time
    int32_t sms;
    FastDiv group;           // query heads of a kv head
};
cudaError_t launch_kv_plan(const sim_kv &kv, const sim_kv_batch &b, cudaStream_t st);
cudaError_t launch_kv_attend(const sim_kv &kv, const sim_kv_batch &b, const KvAttend &a, cudaStream_t st);

// Launch that may begin before the kernel ahead of it in the stream has ended: each kernel waits for that one
// (kv_wait_previous) before it touches memory, so only the launch itself overlaps.
template <typename... Params, typename... Args>
cudaError_t launch_chained(void (*fn)(Params...), int blocks, int threads, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(blocks));
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fn, args...);
}
#ifdef __CUDACC__
__device__ __forceinline__ void kv_wait_previous() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
#endif

int kv_sm_count();  // of the current device

}  // namespace simgb
