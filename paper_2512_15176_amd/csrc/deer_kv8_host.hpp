// Host side of the paged 8-bit KV cache: where its parts lie, launch shapes, argument checks.  A deer_kv8 handle has one of these,
// and so has a context whose target cache is kept in 8 bits.
#pragma once
#include "deer_kv8.hpp"

#include <algorithm>
#include <cmath>

namespace deer {

// Tiles of 32 packed rows whose un-normalised results of a key range the workspace holds: what 512 workgroups of four tiles leave, twice.
constexpr int KV8_PART_TILES = 4096;
constexpr int KV8_WGS = 512;          // workgroups that fill the chip: two per compute unit

struct Kv8Shape { int n_layers, n_q_heads, n_kv_heads, head_dim, max_batch, max_seq, n_pages, max_rows; };

struct Kv8Cache {
    Kv8Shape p{};
    Kv8State st{};
    uint8_t *pages = nullptr;
    float *scales = nullptr, *part = nullptr;
    int *counters = nullptr;
    uint16_t *ring = nullptr, *scratch = nullptr;
    int *ask_start = nullptr, *ask_count = nullptr, *ask_row0 = nullptr;   // requests that the library makes up itself, [max_batch]
    size_t scratch_slots = 0, cache_bytes = 0, work_bytes = 0;
    // the pass
    int batch = 0, rows = 0, max_new = 0, max_len = 0;
    bool long_pass = false;      // rows in the scratch ..
    int scratch_layer = -1;      // .. of this layer

    size_t page_bytes() const { return (size_t)p.n_kv_heads * 2 * KV8_PAGE * p.head_dim; }
    size_t ring_layer() const { return (size_t)p.max_batch * p.n_kv_heads * KV8_SLOTS * p.head_dim; }   // elements of K, and of V
    Kv8Hot ring_view(int layer) const {
        uint16_t *k = ring + 2 * (size_t)layer * ring_layer();
        return Kv8Hot{k, k + ring_layer(), (size_t)p.n_kv_heads * KV8_SLOTS * p.head_dim, (size_t)KV8_SLOTS * p.head_dim, KV8_RING - 1};
    }
    // where the pass's rows of a layer are (the scratch serves one layer after the other)
    Kv8Hot hot_view(int layer) const {
        if (!long_pass) return ring_view(layer);
        return Kv8Hot{scratch, scratch + scratch_slots * p.n_kv_heads * p.head_dim, 0, scratch_slots * p.head_dim, -1};
    }
    uint8_t *layer_pages(int layer) const { return pages + (size_t)layer * p.n_pages * page_bytes(); }
    float *layer_scales(int layer) const { return scales + (size_t)layer * p.n_pages * p.n_kv_heads * 2; }
};

inline const char *check_kv8(const Kv8Shape &p) {
    if (p.n_layers < 1 || p.n_layers > 1024) return "n_layers must be in 1..1024";
    if (p.head_dim != 32 && p.head_dim != 64 && p.head_dim != 128) return "head_dim must be 32, 64 or 128";
    if (p.n_kv_heads < 1 || p.n_kv_heads > 1024 || p.n_q_heads < 1 || p.n_q_heads % p.n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
    if (p.n_q_heads / p.n_kv_heads > 64) return "more than 64 query heads per kv head";
    if (p.max_batch < 1 || p.max_batch > KV8_MAX_BATCH) return "max_batch must be in 1..1024";
    if (p.max_seq < KV8_PAGE || p.max_seq % KV8_PAGE || p.max_seq > 1 << 20) return "max_seq must be a multiple of 64, at most 2^20";
    if (p.n_pages < 1 || p.n_pages > 1 << 24) return "n_pages must be in 1..2^24";
    if (p.max_rows < 1 || p.max_rows > 1 << 20) return "max_rows must be in 1..2^20";
    return nullptr;
}

// Carves the cache (pages, scales, ring, tables) and the workspace (the pass's arrays, scratch, partial results); with null
// bases only the sizes.
inline void plan_kv8(Kv8Cache &c, const Kv8Shape &p, char *cache, char *work) {
    c.p = p;
    size_t off = 0;
    char *base = cache;
    auto take = [&](size_t bytes) { size_t o = off; off = (off + bytes + 255) / 256 * 256; return base ? base + o : nullptr; };
    c.pages = (uint8_t *)take((size_t)p.n_layers * p.n_pages * c.page_bytes());
    c.scales = (float *)take((size_t)p.n_layers * p.n_pages * p.n_kv_heads * 2 * 4);
    c.ring = (uint16_t *)take((size_t)p.n_layers * 2 * c.ring_layer() * 2);
    Kv8State &s = c.st;
    s.max_blocks = p.max_seq / KV8_PAGE; s.max_batch = p.max_batch; s.n_pages = p.n_pages; s.max_rows = p.max_rows;
    s.table = (int *)take((size_t)p.max_batch * s.max_blocks * 4);
    s.len = (int *)take(p.max_batch * 4); s.held = (int *)take(p.max_batch * 4); s.hot = (int *)take(p.max_batch * 4); s.base = (int *)take(p.max_batch * 4);
    s.free = (int *)take((size_t)p.n_pages * 4);
    s.stat = (int *)take(8 * 4);
    c.cache_bytes = off;
    off = 0; base = work;
    s.start = (int *)take(p.max_batch * 4); s.count = (int *)take(p.max_batch * 4); s.hotbase = (int *)take(p.max_batch * 4); s.carry = (int *)take(p.max_batch * 4); s.order = (int *)take(p.max_batch * 4);
    s.cu = (int *)take((p.max_batch + 1) * 4);
    c.ask_start = (int *)take(p.max_batch * 4); c.ask_count = (int *)take(p.max_batch * 4); c.ask_row0 = (int *)take(p.max_batch * 4);
    s.slot = (int *)take((size_t)p.max_rows * 4); s.row_seq = (int *)take((size_t)p.max_rows * 4); s.row_pos = (int *)take((size_t)p.max_rows * 4);
    // a sequence's rows of a long pass touch whole pages: up to 127 slots more than rows
    c.scratch_slots = p.max_rows > KV8_PAGE ? ((size_t)p.max_rows + (size_t)std::min(p.max_batch, p.max_rows) * 127 + 63) / 64 * 64 : 0;
    c.scratch = (uint16_t *)take(2 * c.scratch_slots * p.n_kv_heads * p.head_dim * 2);
    c.counters = (int *)take(KV8_PART_TILES * 4);      // of the items whose key ranges meet: no more than tiles
    c.part = (float *)take((size_t)KV8_PART_TILES * (32 * p.head_dim + 64) * 4);
    c.work_bytes = off;
}

// everything finite, no tokens (masked keys are multiplied by zero weights)
inline hipError_t kv8_clear(Kv8Cache &c, hipStream_t s) {
    hipError_t e = hipMemsetAsync(c.pages, 0, (char *)c.st.table - (char *)c.pages, s);
    if (e == hipSuccess) e = hipMemsetAsync(c.scratch, 0, (char *)c.part - (char *)c.scratch, s);   // and the counters
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_kv8_init, dim3(256), dim3(256), 0, s, c.st);
    c.batch = c.rows = 0;
    return hipGetLastError();
}

inline const char *check_kv8_pass(const Kv8Cache &c, int batch, int rows, int max_new, int max_len) {
    if (batch < 1 || batch > c.p.max_batch) return "batch must be in 1..max_batch";
    if (rows < 0 || rows > c.p.max_rows) return "rows must be in 0..max_rows";
    if (max_new < 0 || max_new > c.p.max_seq) return "max_new must be in 0..max_seq";
    if (max_len < 0 || max_len > c.p.max_seq) return "max_len must be in 0..max_seq";
    if (((long long)max_new * (c.p.n_q_heads / c.p.n_kv_heads) + 31) / 32 > 65535) return "max_new is too large for one pass";
    return nullptr;
}

inline hipError_t kv8_reserve(Kv8Cache &c, hipStream_t s, const int *start, int start_add, const int *count, int count_const, int batch, int rows,
                              int max_new, int max_len) {
    max_new = std::min(max_new, std::max(rows, 0));
    c.batch = batch; c.rows = rows; c.max_new = max_new; c.max_len = max_len;
    c.long_pass = max_new > KV8_PAGE;
    c.scratch_layer = -1;
    // four rows to a thread; a call without rows only gives pages back, up to the batch's tables
    const long long work = rows ? rows : std::min<long long>(c.p.n_pages, (long long)batch * c.st.max_blocks);
    const int wgs = (int)std::max<long long>(1, std::min<long long>(256, (work + 4095) / 4096));
    hipLaunchKernelGGL(k_kv8_reserve, dim3(wgs), dim3(1024), 0, s, c.st, start, start_add, count, count_const, batch, rows, max_new, max_len, c.long_pass ? 1 : 0);
    return hipGetLastError();
}

// pages that a sequence of the pass may touch
inline unsigned kv8_touched(const Kv8Cache &c) { return (unsigned)(c.max_new + KV8_PAGE - 2) / KV8_PAGE + 1; }

template <int HD>
hipError_t kv8_settle_hd(Kv8Cache &c, hipStream_t s, int layer) {
    hipLaunchKernelGGL(k_kv8_settle<HD>, dim3(kv8_touched(c), c.p.n_kv_heads, c.batch), dim3(4 * HD), 0, s, c.st, c.hot_view(layer), c.ring_view(layer), c.long_pass ? 1 : 0,
                       c.layer_pages(layer), c.layer_scales(layer), c.p.n_kv_heads);
    return hipGetLastError();
}
// the pass's rows of the layer are in the hot pages: complete pages go to the pool
inline hipError_t kv8_settle(Kv8Cache &c, hipStream_t s, int layer) {
    if (c.rows == 0 || c.max_new == 0) return hipSuccess;
    return c.p.head_dim == 128 ? kv8_settle_hd<128>(c, s, layer) : c.p.head_dim == 64 ? kv8_settle_hd<64>(c, s, layer) : kv8_settle_hd<32>(c, s, layer);
}

template <int HD, typename T>
hipError_t kv8_append_hd(Kv8Cache &c, hipStream_t s, int layer, const T *k, const T *v, size_t k_stride, size_t v_stride) {
    const Kv8Hot ring = c.ring_view(layer);
    if (c.long_pass) {
        hipLaunchKernelGGL(k_kv8_keep<HD>, dim3(c.p.n_kv_heads, c.batch), dim3(256), 0, s, c.st, ring);
        if (hipError_t e = hipGetLastError()) return e;
    }
    hipLaunchKernelGGL((k_kv8_append<HD, T>), dim3(kv8_touched(c), c.p.n_kv_heads, c.batch), dim3(4 * HD), 0, s, c.st, k, v, k_stride, v_stride, c.hot_view(layer), ring,
                       c.long_pass ? 1 : 0, c.layer_pages(layer), c.layer_scales(layer), c.p.n_kv_heads);
    return hipGetLastError();
}
template <typename T>
hipError_t kv8_append(Kv8Cache &c, hipStream_t s, int layer, const T *k, const T *v, size_t k_stride, size_t v_stride) {
    if (c.rows == 0 || c.max_new == 0) return hipSuccess;
    c.scratch_layer = layer;
    return c.p.head_dim == 128 ? kv8_append_hd<128>(c, s, layer, k, v, k_stride, v_stride)
           : c.p.head_dim == 64 ? kv8_append_hd<64>(c, s, layer, k, v, k_stride, v_stride) : kv8_append_hd<32>(c, s, layer, k, v, k_stride, v_stride);
}

// A pool beyond the memory-side cache (256 MB) is streamed past the L2 where a page has one reader: 16 x 32768 tokens of 8 heads
// of 128 206 -> 186 us, but 16 x 4096, which that cache holds from pass to pass of one layer, 31 -> 34.
constexpr double KV8_SIDE_CACHE = 256e6;

template <typename T>
hipError_t kv8_read(const Kv8Cache &c, hipStream_t s, int layer, const int *seq, const int *pos, int n, T *k, T *v) {
    const size_t items = (size_t)n * (c.p.head_dim / 8);
    hipLaunchKernelGGL(k_kv8_read<T>, dim3((unsigned)((items + 255) / 256), c.p.n_kv_heads), dim3(256), 0, s, c.st, seq, pos, n, c.ring_view(layer), c.layer_pages(layer),
                       c.layer_scales(layer), c.p.n_kv_heads, c.p.head_dim, k, v);
    return hipGetLastError();
}

// What an attention launch takes, in microseconds, by what it streams: k_kv8_attn_few tiles of 16 packed rows x the pages that they see,
// each read by every tile (from L2 and the memory-side cache; fewer workgroups than fill the chip take no less time: 3 sequences, 32
// rows behind 8000 tokens of heads 32 / 8, 384 workgroups 47, k_kv8_attn_many 34); k_kv8_attn_many pages, which a workgroup reads once,
// and tiles of 32 x pages, by the planes that Q and P enter as, with its merge.  The pages are what a row sees on average: a prompt's
// rows half of its own.
// Fitted to 350 calls of bf16 and float32, heads 32 / 8 and 32 / 4 of 128 and 14 / 2 of 64, 1 to 16 sequences of 0 to 16000 tokens, 1 to
// 2000 rows: the choice costs 0.5 % of the better kernel's time on average and 19 % at most.  few / many measured, bf16: heads 32 / 8, 1
// sequence, 32 rows behind 8000 and 16000 tokens 20 / 25, 30 / 31, 200 rows behind 8000 82 / 46; 8 sequences, 8, 17 and 32 rows behind
// 8000 31 / 37, 62 / 45, 83 / 52; 16, 8 and 17 rows behind 16000 127 / 127, 252 / 158; heads 32 / 4, 4 sequences, 17 rows behind
// 16000 60 / 43; heads 14 / 2, 16 sequences, 17 rows behind 2000 and 16000 14 / 16, 47 / 36; prompts, 1 of 500 16 / 19.  Float32: heads
// 32 / 8, 8 sequences, 32 rows behind 2000 and 8000 32 / 56, 97 / 107, prompts, 1 of 1000 and 2000 46 / 57, 125 / 110.
struct Kv8Shares { long long items; int NS; };
inline Kv8Shares kv8_shares(long long items, long long tiles, int pages, int resident) {
    // key ranges: as many as fill the chip (two workgroups of four waves per compute unit), each with eight pages or its waves' four; no more
    // than 32, which the last workgroup adds up (1 sequence of 32768 tokens in 16, 32 and 64 ranges 25.5, 24.7 and 32.9).  257 to 384 items
    // take two where a compute unit holds three workgroups (bf16, heads 32 / 4 of 128, 8 x 17 rows behind 300 .. 3000 tokens 25.1 -> 20.7;
    // 32 / 8, 14 x 12 behind 8000 83 -> 65; float32 heads 14 / 2 of 64, 16 x 21 behind 8000 61 -> 46), but not where it holds two (float32
    // 32 / 4 of 128, 9 x 17 behind 400 .. 3000 28.5 -> 29.4)
    const long long fill = std::max<long long>(KV8_WGS / std::max<long long>(items, 1), resident > 2 && items * 2 <= KV8_WGS / 2 * resident ? 2 : 1);
    return Kv8Shares{items, (int)std::max<long long>(1, std::min<long long>({fill, KV8_PART_TILES / std::max<long long>(tiles, 1), 32, (pages + 7) / 8}))};
}
inline double kv8_few_us(const Kv8Shares &s, double pages, int hd) { return 6.0 + 0.005 * (double)s.items * s.NS + 0.0012 * std::max<double>(s.items, (double)KV8_WGS / s.NS) * pages * hd / 128; }
inline double kv8_many_us(const Kv8Shares &s, long long heads, int rt32, double pages, int hd, int planes) {
    return 10.0 + (0.0008 + (0.0002 + 0.0011 * planes) * rt32) * (double)heads * pages * hd / 128 + (s.NS > 1 ? 5.0 + 0.2 * s.NS : 0.0);
}
// The sequences' order matters where workgroups share compute units.
inline const int *kv8_order(const Kv8Cache &c, long long workgroups) { return c.batch > 1 && c.batch <= KV8_SORT && workgroups > KV8_WGS / 2 ? c.st.order : nullptr; }
template <int HD, int SRC>
hipError_t kv8_attend_src(Kv8Cache &c, hipStream_t s, Kv8Attn &a) {
    const int B = c.batch, packed = c.max_new * a.G, pages = (c.max_len + KV8_PAGE - 1) / KV8_PAGE;
    const int rt16 = (packed + 15) / 16, rt32 = (packed + 31) / 32, groups = (rt32 + 3) / 4;
    const long long heads = (long long)B * a.Hkv;
    const Kv8Shares f = kv8_shares(heads * rt16, heads * rt16, pages, kv8_few_resident<HD, SRC>());
    const Kv8Shares m = kv8_shares(heads * groups, heads * rt32, pages * 2, 2);      // (a workgroup of this kernel takes four pages at least)
    const double seen = (c.max_len - 0.5 * c.max_new) / KV8_PAGE + 0.5;
    if (kv8_few_us(f, seen, HD) <= kv8_many_us(m, heads, rt32, seen, HD, Kv8Planes<HD, SRC>::N) && rt16 <= 65535) {
        a.rts = rt16; a.NS = f.NS; a.order = kv8_order(c, f.items * f.NS);
        const dim3 grid(a.Hkv * a.NS, rt16, B);
        if (rt16 == 1 && (double)c.p.n_layers * B * pages * c.page_bytes() > KV8_SIDE_CACHE) hipLaunchKernelGGL((k_kv8_attn_few<HD, SRC, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_kv8_attn_few<HD, SRC, false>), grid, dim3(256), 0, s, a);
        return hipGetLastError();
    }
    a.rts = rt32; a.NS = m.NS; a.order = kv8_order(c, m.items * m.NS);
    hipLaunchKernelGGL((k_kv8_attn_many<HD, SRC>), dim3(a.Hkv * a.NS, groups, B), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.NS > 1) hipLaunchKernelGGL((k_kv8_merge<HD, SRC>), dim3(a.Hkv, rt32, B), dim3(4 * HD), 0, s, a);
    return hipGetLastError();
}
// a: what the caller knows (limits, q, out or fragments)
template <int SRC>
hipError_t kv8_attend(Kv8Cache &c, hipStream_t s, int layer, Kv8Attn a, double scale) {
    if (c.rows == 0 || c.max_new == 0) return hipSuccess;
    a.s = c.st; a.hot = c.hot_view(layer); a.pages = c.layer_pages(layer); a.scales = c.layer_scales(layer);
    a.part = c.part; a.counters = c.counters; a.Hq = c.p.n_q_heads; a.Hkv = c.p.n_kv_heads; a.G = a.Hq / a.Hkv;
    a.scale_log2e = (float)(scale * 1.4426950408889634);
    a.m_init = -3e38f / std::max(1.f, a.scale_log2e);     // times scale_log2e it stays finite
    return c.p.head_dim == 128 ? kv8_attend_src<128, SRC>(c, s, a) : c.p.head_dim == 64 ? kv8_attend_src<64, SRC>(c, s, a) : kv8_attend_src<32, SRC>(c, s, a);
}

}  // namespace deer
