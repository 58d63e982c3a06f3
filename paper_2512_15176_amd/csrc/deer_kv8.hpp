// Device code of the paged 8-bit KV cache: the tables of a pass, the append that fills pages, the attention that reads them.
//
// A page is 64 tokens of one sequence.  A complete page holds, per layer and kv head, e4m3 keys and values and one scale for
// each: s = 2^e, the smallest power of two with amax / s <= 448 (amax over the page's 64 x head_dim values of that head).  With a
// power of two x / s and x8 * s are exact and x8 * s is a bf16, so that a page's content is a function of its bf16 rows alone;
// what it costs against amax / 448 is up to one of the 14 binades between the largest value and e4m3's first subnormal.
//
// A row reads the pages before its own in 8 bits and its own page (that of the last key it sees) in bf16, as the rows came.  What
// a row reads thus depends on positions alone: a block of k rows equals k single rows, a prompt equals its tokens one by one, and a
// page that rejected drafts had completed is quantised again when it next fills.
//
// The bf16 rows ("hot" pages) are in one of two places, both in the order of the bf16 caches (k_cache_off / v_cache_off):
//   ring     128 slots per layer, sequence and kv head: the open page and the one before or behind it; passes of up to 64 rows per
//            sequence write there (slot = position mod 128).  64 slots more keep the page in which the last longer pass started, so
//            that it can be taken back.
//   scratch  one layer's rows of a longer pass, the pages that it touches packed one after the other; the last two go to the ring.
// Ring and scratch are addressed as (position + hotbase[sequence]) & mask.
//
// A page's 8-bit rows lie in the order of the bf16 fragments (see k_cache_off), two fragments to a chunk of 64 lanes x 16 bytes: lane's
// bytes 0..7 are its eight elements of fragment 2c, bytes 8..15 those of 2c + 1.  A wave reads a chunk as one contiguous 1 KB.
#pragma once
#include "deer_kernels.hpp"

namespace deer {

constexpr int KV8_PAGE = 64, KV8_RING = 128, KV8_SLOTS = 192;   // slots of the ring, and with the kept page
constexpr int KV8_MAX_BATCH = 1024;
constexpr int KV8_SORT = 128;     // sequences that a pass puts in order

struct Kv8State {      // device arrays
    int *table;        // [max_batch][max_blocks]: page of every 64 tokens, -1 beyond the pages held
    int *len, *held, *hot;         // [max_batch]: tokens, pages, first page whose bf16 rows the ring holds
    int *base;         // [max_batch]: the kept page holds the tokens of its page before this position
    int *free;         // [n_pages]: stack of free pages
    int *stat;         // 0 free pages, 1 sequences refused by the last call, 2 arrival counter
    // the pass
    int *start, *count, *hotbase;  // [max_batch]: first position, rows granted, see above
    int *carry;        // [max_batch]: where the open page's older rows are: 0 none, 1 the ring, 2 the kept page
    int *cu;           // [max_batch + 1]: first row of every sequence
    int *order;        // [max_batch]: passes of up to KV8_SORT sequences: those with the most keys first
    int *slot, *row_seq, *row_pos; // [max_rows]
    int max_blocks, max_batch, n_pages, max_rows;
};

struct Kv8Hot {        // bf16 rows of one layer
    uint16_t *k, *v;
    size_t seq_stride, head_stride;   // elements
    int mask;
};

// ------------------------------------------------------------------------------------------
// tables of a pass
// ------------------------------------------------------------------------------------------
// Inclusive sums of two pairs of numbers (each below 2^31) over 1024 threads, in one pass; tmp: LDS
struct Kv8Sums { unsigned long long a, b; };
__device__ __forceinline__ unsigned long long kv8_up(unsigned long long v, int off, int lane) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute((lane - off) << 2, (int)(uint32_t)v);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_ds_bpermute((lane - off) << 2, (int)(uint32_t)(v >> 32));
    return lane >= off ? ((unsigned long long)hi << 32) | lo : 0ull;
}
__device__ __forceinline__ Kv8Sums kv8_scan(Kv8Sums v, Kv8Sums (&tmp)[16]) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) { v.a += kv8_up(v.a, off, lane); v.b += kv8_up(v.b, off, lane); }
    if (lane == 63) tmp[w] = v;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 15; ++i)
        if (i < w) { v.a += tmp[i].a; v.b += tmp[i].b; }
    return v;
}

// number of entries of the ascending a[0 .. n) that are <= x
__device__ __forceinline__ int kv8_upper(const int *a, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) { const int mid = (lo + hi) >> 1; if (a[mid] <= x) lo = mid + 1; else hi = mid; }
    return lo;
}

__global__ void k_kv8_init(Kv8State s) {
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x, n = (size_t)gridDim.x * blockDim.x;
    for (size_t j = i; j < (size_t)s.max_batch * s.max_blocks; j += n) s.table[j] = -1;
    for (size_t j = i; j < (size_t)s.n_pages; j += n) s.free[j] = s.n_pages - 1 - (int)j;
    for (size_t j = i; j < (size_t)s.max_batch; j += n) { s.len[j] = s.held[j] = s.hot[j] = s.base[j] = s.start[j] = s.count[j] = s.hotbase[j] = s.carry[j] = 0; s.order[j] = (int)j; }
    for (size_t j = i; j <= (size_t)s.max_batch; j += n) s.cu[j] = 0;
    for (size_t j = i; j < (size_t)s.max_rows; j += n) { s.slot[j] = -1; s.row_seq[j] = -1; s.row_pos[j] = 0; }
    if (i < 8) s.stat[i] = i == 0 ? s.n_pages : 0;
}

// Sequence b keeps its first start tokens and takes count rows behind them; afterwards it holds ceil((start + count) / 64) pages.
// Pages given back go on the stack before any is taken from it, such that releases followed by the same requests give the same
// table: taken page i is the i-th page given back (in order of sequence and block), then the stack's top and down.
// A sequence is refused (keeps its pages and tokens, gets no rows) for numbers out of range, a start behind its tokens, a start
// inside a page whose bf16 rows are gone, or, like every growing one behind it, where the pages do not suffice.
// Every workgroup works out all sequences (one scan) and writes its share of table entries and rows, four rows to a thread; the
// state itself is written by the last to arrive, when all have read it (so that start may be the lengths themselves), with the order of up
// to 128 sequences by their keys, in which attention takes them.  Bound by latency:
// 16 sequences 4 to 6 us, 1000 prompts with 512500 rows 13 us (their 6.1 MB would take 1).  grid: any; 1024 threads; B <= 1024.
__global__ __launch_bounds__(1024) void k_kv8_reserve(Kv8State s, const int *start, int start_add, const int *__restrict__ count,
                                                      int count_const, int B, int rows, int max_new, int max_len, int scratch) {
    __shared__ int s_row[KV8_MAX_BATCH], s_start[KV8_MAX_BATCH], s_n[KV8_MAX_BATCH], s_held[KV8_MAX_BATCH], s_tp[KV8_MAX_BATCH],
        s_grow[KV8_MAX_BATCH], s_give[KV8_MAX_BATCH], s_keys[KV8_SORT], s_taken, s_given, s_refused, s_flag;
    __shared__ Kv8Sums tmp[16];
    const int b = threadIdx.x;
    int st = 0, n = 0, len = 0, held = 0, hot = 0, base = 0;
    if (b < B) {
        st = (start ? start[b] : 0) + start_add;
        n = count ? count[b] : count_const;
        len = s.len[b]; held = s.held[b]; hot = s.hot[b]; base = s.base[b];
    }
    const int top = s.stat[0];
    if (b == 0) { s_taken = 0; s_given = 0; s_refused = 0; }
    const int rn = b < B ? min(max(n, 0), rows) : 0;              // the rows' layout follows the request, granted or not
    const bool in_ring = st / KV8_PAGE >= hot, kept = st / KV8_PAGE == base / KV8_PAGE && st <= base;
    bool ok = b < B && st >= 0 && n >= 0 && n <= max_new && st <= max_len && st + n <= max_len && st <= len && ((st & (KV8_PAGE - 1)) == 0 || in_ring || kept);
    const int tp = ok ? (st + n + KV8_PAGE - 1) / KV8_PAGE : held, first = st / KV8_PAGE;
    const int grow = max(0, tp - held), give = max(0, held - tp), touched = ok && n > 0 ? (st + n - 1) / KV8_PAGE - first + 1 : 0;
    const Kv8Sums v = kv8_scan(Kv8Sums{((unsigned long long)rn << 32) | (unsigned)touched, ((unsigned long long)grow << 32) | (unsigned)give}, tmp);
    const int row_end = (int)(v.a >> 32), row0 = row_end - rn, touched_end = (int)(uint32_t)v.a, grow_end = (int)(v.b >> 32), give_end = (int)(uint32_t)v.b;
    // A sequence whose rows end behind the last is refused, and so is every one behind it: what they would give or take lies behind
    // everybody's in the sums, and counts for nobody.
    ok = ok && row_end <= rows;
    if (ok) atomicMax(&s_given, give_end);
    __syncthreads();
    const int given = s_given, avail = top + given;
    if (grow > 0 && grow_end > avail) ok = false;
    const int m = ok ? n : 0, last = (st + max(m, 1) - 1) / KV8_PAGE;
    s_row[b] = b < B ? row0 : 0x7fffffff; s_start[b] = st; s_n[b] = m; s_held[b] = held; s_tp[b] = tp; s_grow[b] = grow_end; s_give[b] = give_end;
    if (b < KV8_SORT) s_keys[b] = m > 0 ? st + m : 0;
    if (ok && grow > 0) atomicMax(&s_taken, grow_end);
    if (b < B && !ok) atomicAdd(&s_refused, 1);
    __syncthreads();
    const int taken = s_taken;
    auto back = [&](int i) {      // the table entry of the i-th page given back
        const int q = kv8_upper(s_give, KV8_MAX_BATCH, i);
        return s.table + (size_t)q * s.max_blocks + s_tp[q] + i - (q ? s_give[q - 1] : 0);
    };
    auto take = [&](int i) { return i < given ? *back(i) : s.free[top - 1 - (i - given)]; };
    const int tid = blockIdx.x * 1024 + threadIdx.x, nth = gridDim.x * 1024;
    for (int r0 = tid * 4; r0 < rows; r0 += nth * 4) {
        int q = kv8_upper(s_row, B, r0) - 1, at = -1, page = 0;      // at: the table entry that `page` is
        int sl[4], sq[4], ps[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = r0 + e;
            while (q + 1 < B && s_row[q + 1] <= r) ++q;
            sl[e] = sq[e] = -1; ps[e] = 0;
            if (q >= 0 && r - s_row[q] < s_n[q]) {
                ps[e] = s_start[q] + r - s_row[q]; sq[e] = q;
                const int pi = ps[e] / KV8_PAGE, entry = q * s.max_blocks + pi;      // (fits: 1024 sequences of 2^14 pages)
                if (entry != at) {
                    at = entry;
                    page = pi < s_held[q] ? s.table[entry] : take((q ? s_grow[q - 1] : 0) + pi - s_held[q]);
                }
                if (ps[e] % KV8_PAGE == 0 && pi >= s_held[q]) s.table[entry] = page;      // (a page that is taken starts with a row of the pass)
                sl[e] = page * KV8_PAGE + ps[e] % KV8_PAGE;
            }
        }
        if (r0 + 4 <= rows) {
            *(int4 *)(s.slot + r0) = make_int4(sl[0], sl[1], sl[2], sl[3]);
            *(int4 *)(s.row_seq + r0) = make_int4(sq[0], sq[1], sq[2], sq[3]);
            *(int4 *)(s.row_pos + r0) = make_int4(ps[0], ps[1], ps[2], ps[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (r0 + e < rows) { s.slot[r0 + e] = sl[e]; s.row_seq[r0 + e] = sq[e]; s.row_pos[r0 + e] = ps[e]; }
        }
    }
    for (int j = tid; j < given - taken; j += nth) {      // pages that nobody takes: their entries, and the stack's from `top` on, are read by nobody else
        int *entry = back(given - 1 - j);
        s.free[top + j] = *entry;
        *entry = -1;
    }
    if (gridDim.x > 1) { if (!arrive_last(&s.stat[2], gridDim.x, &s_flag)) return; }
    else __syncthreads();
    if (b < B) {
        s.start[b] = st; s.count[b] = m; s.cu[b] = min(row0, rows);
        s.hotbase[b] = scratch ? (touched_end - touched - first) * KV8_PAGE : 0;
        if (b == B - 1) s.cu[B] = min(row_end, rows);
        if (B > 1 && B <= KV8_SORT) {
            const int mine = s_keys[b];
            int at = 0;
            for (int j = 0; j < B; ++j) at += s_keys[j] > mine || (s_keys[j] == mine && j < b) ? 1 : 0;
            s.order[at] = b;
        }
        const int older = m > 0 && st % KV8_PAGE ? (in_ring ? 1 : 2) : 0;
        s.carry[b] = scratch || older == 2 ? older : 0;       // (a short pass finds the ring's rows where they are)
        if (ok) {
            s.len[b] = st + n; s.held[b] = tp;
            // (without rows, back inside the kept page: the ring does not hold it)
            s.hot[b] = n > 0 ? max(min(hot, first), last - 1) : st % KV8_PAGE && !in_ring ? hot : min(hot, first);
            s.base[b] = (scratch && older) || (kept && st % KV8_PAGE) ? st : st < base ? first * KV8_PAGE : base;
        }
    }
    for (int i = b; i < min(given, taken); i += 1024) *back(i) = -1;
    if (b == 0) { s.stat[0] = top + given - taken; s.stat[1] = s_refused; }
}

// The requests of a prompt pass, from its attention tiles (see PassRows; the tiles of a sequence follow each other): sequences
// without a tile keep what they hold.  row0: attention row of a sequence's first.  One workgroup of 1024.
__global__ __launch_bounds__(1024) void k_kv8_prompt_pass(const int4 *__restrict__ desc, int n_desc, const int *__restrict__ len, int B, int *__restrict__ start,
                                                          int *__restrict__ count, int *__restrict__ row0) {
    for (int b = threadIdx.x; b < B; b += 1024) { start[b] = len[b]; count[b] = 0; row0[b] = 0; }
    __syncthreads();
    for (int t = threadIdx.x; t < n_desc; t += 1024) {
        const int4 d = desc[t];
        if (t == 0 || desc[t - 1].x != d.x) {
            int n = 0;
            for (int u = t; u < n_desc && desc[u].x == d.x; ++u) n += desc[u].z & 63;
            start[d.x] = d.y; count[d.x] = n; row0[d.x] = t * 32;
        }
    }
}
// The request of one sequence; the others keep what they hold.
__global__ void k_kv8_one(const int *__restrict__ len, int B, int b, int first, int n, int *__restrict__ start, int *__restrict__ count) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < B) { start[i] = i == b ? first : len[i]; count[i] = i == b ? n : 0; }
}

// ------------------------------------------------------------------------------------------
// append
// ------------------------------------------------------------------------------------------
template <typename SrcT>
__device__ __forceinline__ uint4 load8_bf16(const SrcT *p);
template <>
__device__ __forceinline__ uint4 load8_bf16<uint16_t>(const uint16_t *p) { return *(const uint4 *)p; }
template <>
__device__ __forceinline__ uint4 load8_bf16<float>(const float *p) {
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    return pack8(v);
}
// whether one of eight bf16 is an infinity or NaN
__device__ __forceinline__ bool nonfinite8(uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) bad = bad || (w[e] & 0x7f800000u) == 0x7f800000u || (w[e] & 0x7f80u) == 0x7f80u;
    return bad;
}

// the scale of a page whose largest magnitude is amax: 2^e, smallest with amax <= 448 * 2^e = 1.75 * 2^(e + 8); 1 for a page of
// zeros.  Not below 2^-100: what is smaller than 2^-109 then becomes zero.
__device__ __forceinline__ float kv8_scale(float amax) {
    if (!(amax > 0.f)) return 1.f;
    const uint32_t u = __float_as_uint(amax);
    const int e = max((int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), -100);
    return __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ float finite_abs(float x) { x = fabsf(x); return x < INFINITY ? x : 0.f; }
__device__ __forceinline__ float amax8(float a, uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) a = fmaxf(a, fmaxf(finite_abs(bf2f(w[e] & 0xffffu)), finite_abs(__uint_as_float(w[e] & 0xffff0000u))));
    return a;
}
// eight bf16 times inv (a power of two) as e4m3, nearest even
__device__ __forceinline__ uint2 quant8(uint4 v, float inv) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    int o[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(bf2f(w[2 * e] & 0xffffu) * inv, __uint_as_float(w[2 * e] & 0xffff0000u) * inv, 0, false);
        o[e] = __builtin_amdgcn_cvt_pk_fp8_f32(bf2f(w[2 * e + 1] & 0xffffu) * inv, __uint_as_float(w[2 * e + 1] & 0xffff0000u) * inv, p, true);
    }
    return make_uint2((uint32_t)o[0], (uint32_t)o[1]);
}
// A page's 64 rows of one head in registers, K and V in fragment order: thread t of 4 HD has the two fragments' vectors of chunk t / 64
// that belong to lane t % 64.  They are quantised into the pool; all threads call it.
template <int HD>
__device__ __forceinline__ void kv8_quantise(const uint4 (&x)[2][2], uint8_t *__restrict__ pp, float *__restrict__ scales, float (&s_max)[2][HD / 16]) {
    constexpr int W = HD / 16;      // waves
    float amax[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        amax[kv] = amax8(amax8(0.f, x[kv][0]), x[kv][1]);
        amax[kv] = fmaxf(amax[kv], dppf<0xB1>(amax[kv]));      // (see dpp: sixteen lanes, then the four groups)
        amax[kv] = fmaxf(amax[kv], dppf<0x4E>(amax[kv]));
        amax[kv] = fmaxf(amax[kv], dppf<0x141>(amax[kv]));
        amax[kv] = fmaxf(amax[kv], dppf<0x140>(amax[kv]));
        amax[kv] = fmaxf(amax[kv], shx(amax[kv], 16));
        amax[kv] = fmaxf(amax[kv], shx(amax[kv], 32));
        if ((threadIdx.x & 63) == 0) s_max[kv][threadIdx.x >> 6] = amax[kv];
    }
    __syncthreads();
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        float m = s_max[kv][0];
#pragma unroll
        for (int i = 1; i < W; ++i) m = fmaxf(m, s_max[kv][i]);
        const float sc = kv8_scale(m);
        const float inv = __uint_as_float((254u << 23) - __float_as_uint(sc));    // 1 / 2^e
        if (threadIdx.x == 0) scales[kv] = sc;
        const uint2 a = quant8(x[kv][0], inv), d = quant8(x[kv][1], inv);
        *(uint4 *)(pp + (size_t)kv * KV8_PAGE * HD + (size_t)threadIdx.x * 16) = make_uint4(a.x, a.y, d.x, d.y);
    }
}

// Where a page of a sequence and head lies.
struct Kv8At { size_t hot, ring, kept; };      // elements
__device__ __forceinline__ Kv8At kv8_at(const Kv8State &s, const Kv8Hot &hot, const Kv8Hot &ring, int b, int head, int page, int hd) {
    const size_t rb = (size_t)b * ring.seq_stride + (size_t)head * ring.head_stride;
    return Kv8At{(size_t)b * hot.seq_stride + (size_t)head * hot.head_stride + (size_t)((page * KV8_PAGE + s.hotbase[b]) & hot.mask) * hd,
                 rb + (size_t)((page * KV8_PAGE) & ring.mask) * hd, rb + (size_t)KV8_RING * hd};
}

// A long pass that starts inside a page: the page's rows go from the ring to the kept page (the pass's last pages may take that half of
// the ring, and the pass may be taken back).  grid: x kv head, y sequence; 256 threads
template <int HD>
__global__ __launch_bounds__(256) void k_kv8_keep(Kv8State s, Kv8Hot ring) {
    const int b = blockIdx.y, head = blockIdx.x;
    if (s.carry[b] != 1) return;
    const Kv8At at = kv8_at(s, ring, ring, b, head, s.start[b] / KV8_PAGE, HD);
    for (int i = threadIdx.x * 8; i < KV8_PAGE * HD; i += 256 * 8) {
        *(uint4 *)(ring.k + at.kept + i) = *(const uint4 *)(ring.k + at.ring + i);
        *(uint4 *)(ring.v + at.kept + i) = *(const uint4 *)(ring.v + at.ring + i);
    }
}

// Rows of the pass [row][kv head][head_dim] enter the cache, one page of one head per workgroup: the rows become fragments (K's are the
// rows' own octets; V goes through LDS, as a fragment has eight tokens of a channel), the page's older rows join them from the ring
// or, behind a long pass's start or a pass taken back, from the kept page; the fragments go to the hot page, to the ring if the pass is long
// and the page one of its last two, and, quantised, to the pool if the page is complete.
// A token with an infinity or NaN in its K or V row of a head gets a key of NaNs and a value of zeros there: rows that see it come out
// NaN, and rows that do not, whose weight for it is zero, do not meet 0 x NaN.
// Bound by latency: everything that is read is asked for before anything is waited for (16 sequences x 32 rows, 8 heads of 128:
// 9 us, the launch's 2 and 7 for tables, rows, LDS and stores; a prompt of 4096 rows, 42 MB, 15 us).
// grid: x page of the sequence's pass, y kv head, z sequence; 4 HD threads
template <int HD, typename SrcT>
__global__ __launch_bounds__(4 * HD) void k_kv8_append(Kv8State s, const SrcT *__restrict__ k, const SrcT *__restrict__ v, size_t k_stride, size_t v_stride,
                                                       Kv8Hot hot, Kv8Hot ring, int is_long, uint8_t *__restrict__ pages, float *__restrict__ scales, int Hkv) {
    constexpr int OCTS = HD / 8, VS = HD + 8;       // padded row of V in LDS
    __shared__ __attribute__((aligned(16))) uint16_t s_v[KV8_PAGE * VS];
    __shared__ int s_bad[KV8_PAGE];
    __shared__ float s_max[2][HD / 16];
    const int b = blockIdx.z, head = blockIdx.y, n = s.count[b];
    if (n == 0) return;
    const int st = s.start[b], end = st + n, first = st / KV8_PAGE, last = (end - 1) / KV8_PAGE, page = first + blockIdx.x;
    if (page > last) return;
    const int t0 = max(st - page * KV8_PAGE, 0), t1 = min(end - page * KV8_PAGE, KV8_PAGE);    // the page's rows of this pass
    const int row0 = s.cu[b] + page * KV8_PAGE - st;       // row of the page's token 0
    const bool whole = t1 == KV8_PAGE, out = is_long && page >= last - 1;
    const int carry = t0 > 0 ? s.carry[b] : 0;             // (0: the older rows are where they belong)
    const Kv8At at = kv8_at(s, hot, ring, b, head, page, HD);
    const size_t older = carry ? at.kept : at.ring;        // carry: the pass is long (kept by k_kv8_keep), or taken back
    const int id = whole ? s.table[(size_t)b * s.max_blocks + page] : -1;
    // V: the rows' octets, two to a thread
    uint4 xv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int tok = (threadIdx.x + 4 * HD * i) / OCTS, oct = threadIdx.x % OCTS;
        xv[i] = make_uint4(0u, 0u, 0u, 0u);
        if (tok >= t0 && tok < t1) xv[i] = load8_bf16(v + (size_t)(row0 + tok) * v_stride + (size_t)head * HD + oct * 8);
    }
    // K in fragment order, and what is older of V's fragments
    const int lane = threadIdx.x & 63, f0 = (threadIdx.x >> 6) * 2, rr = lane & 31, half = lane >> 5, blk = f0 / (HD / 16) * 32;
    const int tok = blk + 16 * ((rr >> 2) & 1) + 4 * (rr >> 3) + (rr & 3);      // of a K vector
    const bool mine = tok >= t0 && tok < t1, before = tok < t0;
    uint4 x[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int f = f0 + u, oct = f % (HD / 16) * 2 + half, tok0 = blk + 16 * half + 8 * u;     // tok0: the first of a V vector's eight tokens
        const size_t off = ((size_t)f * 64 + lane) * 8;
        x[0][u] = x[1][u] = make_uint4(0u, 0u, 0u, 0u);
        if (mine) x[0][u] = load8_bf16(k + (size_t)(row0 + tok) * k_stride + (size_t)head * HD + oct * 8);
        else if (before && (whole || carry)) x[0][u] = *(const uint4 *)(ring.k + older + off);
        if (tok0 < t0 && (tok0 + 8 > t0 || whole || carry)) x[1][u] = *(const uint4 *)(ring.v + older + off);
    }
    if (threadIdx.x < KV8_PAGE) s_bad[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int vt = (threadIdx.x + 4 * HD * i) / OCTS, oct = threadIdx.x % OCTS;
        if (nonfinite8(xv[i])) s_bad[vt] = 1;
        *(uint4 *)(s_v + vt * VS + oct * 8) = xv[i];
    }
    if (mine && (nonfinite8(x[0][0]) || nonfinite8(x[0][1]))) s_bad[tok] = 1;
    __syncthreads();
    const bool bad = mine && s_bad[tok];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int f = f0 + u, ch = f % (HD / 16) / 2 * 32 + rr, tok0 = blk + 16 * half + 8 * u;
        const size_t off = ((size_t)f * 64 + lane) * 8;
        if (bad) x[0][u] = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
        if (mine || (before && carry)) {
            *(uint4 *)(hot.k + at.hot + off) = x[0][u];
            if (out) *(uint4 *)(ring.k + at.ring + off) = x[0][u];
        }
        const bool some = tok0 < t1 && tok0 + 8 > t0;
        if (some) {      // eight tokens of a channel
            uint32_t w[4] = {x[1][u].x, x[1][u].y, x[1][u].z, x[1][u].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int tk = tok0 + e;
                const uint32_t y = tk >= t0 && tk < t1 && !s_bad[tk] ? s_v[tk * VS + ch] : tk < t0 ? (w[e >> 1] >> (16 * (e & 1))) & 0xffffu : 0u;
                w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | y << 16 : (w[e >> 1] & 0xffff0000u) | y;
            }
            x[1][u] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (some || (tok0 < t0 && carry)) {
            *(uint4 *)(hot.v + at.hot + off) = x[1][u];
            if (out) *(uint4 *)(ring.v + at.ring + off) = x[1][u];
        }
    }
    if (!whole) return;      // (the whole workgroup)
    if ((unsigned)id >= (unsigned)s.n_pages) return;
    const size_t pg = (size_t)id * Hkv + head;
    kv8_quantise<HD>(x, pages + pg * (2 * KV8_PAGE * HD), scales + pg * 2, s_max);
}

// Where another kernel has put the pass's rows into the hot pages (the engine's QKV projection): pages that they complete go to the pool,
// and with the rows in the scratch (is_long) the last two pages to the ring.  grid as above
template <int HD>
__global__ __launch_bounds__(4 * HD) void k_kv8_settle(Kv8State s, Kv8Hot hot, Kv8Hot ring, int is_long, uint8_t *__restrict__ pages, float *__restrict__ scales, int Hkv) {
    __shared__ float s_max[2][HD / 16];
    const int b = blockIdx.z, head = blockIdx.y, n = s.count[b];
    if (n == 0) return;
    const int st = s.start[b], end = st + n, first = st / KV8_PAGE, last = (end - 1) / KV8_PAGE, page = first + blockIdx.x;
    if (page > last) return;
    const bool whole = end >= (page + 1) * KV8_PAGE, out = is_long && page >= last - 1;
    if (!whole && !out) return;
    const Kv8At at = kv8_at(s, hot, ring, b, head, page, HD);
    const int id = whole ? s.table[(size_t)b * s.max_blocks + page] : -1;
    uint4 x[2][2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const size_t off = ((size_t)((threadIdx.x >> 6) * 2 + u) * 64 + (threadIdx.x & 63)) * 8;
            x[kv][u] = *(const uint4 *)((kv ? hot.v : hot.k) + at.hot + off);
            if (out) *(uint4 *)((kv ? ring.v : ring.k) + at.ring + off) = x[kv][u];
        }
    if (!whole) return;
    if ((unsigned)id >= (unsigned)s.n_pages) return;
    const size_t pg = (size_t)id * Hkv + head;
    kv8_quantise<HD>(x, pages + pg * (2 * KV8_PAGE * HD), scales + pg * 2, s_max);
}

// Rows as they stand in the cache (complete pages in 8 bits, else bf16) for n (sequence, position) pairs; zeros for a pair that names no
// token.  One thread per (row, octet) of a head: the bytes of 16 tokens of a channel are one 16-byte vector, so that the tokens of a
// workgroup, which mostly follow each other, find theirs in the lines that the first has fetched.  (As vectors, turned in LDS, 4096
// rows of 8 heads of 128 took as long, 13 us, and 512 rows in no order 20 instead of 5.)  grid: x rows, y head
template <typename DstT>
__global__ __launch_bounds__(256) void k_kv8_read(Kv8State s, const int *__restrict__ seq, const int *__restrict__ pos, int n, Kv8Hot ring,
                                                  const uint8_t *__restrict__ pages, const float *__restrict__ scales, int Hkv, int hd,
                                                  DstT *__restrict__ k, DstT *__restrict__ v) {
    const int octs = hd >> 3, head = blockIdx.y;
    const size_t gid = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (gid >= (size_t)n * octs) return;
    const int oct = (int)(gid % octs), r = (int)(gid / octs);
    const int b = seq[r], ps = pos[r];
    float kf[8], vf[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) kf[e] = vf[e] = 0.f;
    if (b >= 0 && b < s.max_batch && ps >= 0 && ps < s.len[b]) {
        const int page = ps / KV8_PAGE;
        if ((page + 1) * KV8_PAGE <= s.len[b]) {
            const int id = s.table[(size_t)b * s.max_blocks + page];
            if ((unsigned)id < (unsigned)s.n_pages) {
                const size_t at = (size_t)id * Hkv + head;
                const uint8_t *pp = pages + at * (2 * KV8_PAGE * hd);
                const float ks = scales[at * 2], vs = scales[at * 2 + 1];
                auto byte_of = [](size_t elem) {   // the bf16 order's element -> the chunk order's byte
                    const size_t f = elem >> 9, lane = (elem >> 3) & 63;
                    return (f >> 1) * 1024 + lane * 16 + (f & 1) * 8 + (elem & 7);
                };
                const uint2 kr = *(const uint2 *)(pp + byte_of(k_cache_off(ps % KV8_PAGE, oct, hd)));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t vb = pp[(size_t)KV8_PAGE * hd + byte_of(v_cache_off(ps % KV8_PAGE, oct * 8 + e, hd))];
                    kf[e] = __builtin_amdgcn_cvt_f32_fp8((int)((e < 4 ? kr.x : kr.y) >> (8 * (e & 3))), 0) * ks;
                    vf[e] = __builtin_amdgcn_cvt_f32_fp8((int)vb, 0) * vs;
                }
            }
        } else {
            const int slot = page >= s.hot[b] ? ps & ring.mask : KV8_RING + ps % KV8_PAGE;
            const size_t base = (size_t)b * ring.seq_stride + (size_t)head * ring.head_stride;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                kf[e] = bf2f(ring.k[base + k_cache_off(slot, oct, hd) + e]);
                vf[e] = bf2f(ring.v[base + v_cache_off(slot, oct * 8 + e, hd)]);
            }
        }
    }
    const size_t o = ((size_t)r * Hkv + head) * hd + oct * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (sizeof(DstT) == 2) { k[o + e] = (DstT)f2bf(kf[e]); v[o + e] = (DstT)f2bf(vf[e]); }
        else { k[o + e] = kf[e]; v[o + e] = vf[e]; }
    }
}

// ------------------------------------------------------------------------------------------
// attention
//   The rows of a sequence and the query heads of a kv head are packed: packed row m = row * G + g, G = Hq / Hkv, so that one token
//   of a group of four fills four of a tile's 32 operand rows and a block of 32 fills four tiles.  S^T = K Q^T and O^T = V^T P^T as
//   in k_attn; e4m3 becomes bf16 (exactly, with the page's scale) on its way to the matrix instruction.
//   Q and P enter as NQ and NP bf16 planes: one where q and the result are bf16 (q is exact; P is rounded by at most 2^-9 of itself,
//   less than the result's own rounding), three for float32 (24 bits).  The engine's fragments: one for a dense model, as the low
//   plane of its Q would add nine bits to scores whose keys have four (verify pass of 12 layers of the 8B model, 16 x 32768 tokens:
//   12.2 ms with both planes, 10.3 with one); two for a mixture, whose rows that lie between two experts go to the other one after
//   any rounding (one plane: a row of the tests did, and its logits were 0.1 off).
// ------------------------------------------------------------------------------------------
enum { KV8_BF16 = 0, KV8_F32 = 1, KV8_FRAG = 2, KV8_FRAG2 = 3 };   // where q comes from and the result goes: rows, or the engine's fragments

struct Kv8Attn {
    Kv8State s;
    Kv8Hot hot;
    const uint8_t *pages; const float *scales;     // the layer's
    const int *limits;                             // keys that a row sees, or null: its position + 1
    const void *q; void *out;                      // rows
    long long q_stride, out_stride;                // elements
    const uint4 *qhi, *qlo; uint4 *xhi, *xlo;      // fragments
    const int *q_row0;                             // fragments: attention row of a sequence's first row; null: 32 * sequence
    float *part; int *counters;                    // counters: zero between kernels
    const int *order;                              // sequence of the grid's z, or null: z
    int Hq, Hkv, G, NS, rts;                       // NS key ranges; rts: tiles of packed rows per sequence
    float scale_log2e, m_init;
};

template <int N>
__device__ __forceinline__ void split_planes(const float *v, uint4 (&o)[N]) {
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
    for (int p = 0; p < N; ++p) {
        uint32_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = f2bf2(r[2 * e], r[2 * e + 1]);
            if (p + 1 < N) { r[2 * e] -= __uint_as_float(h[e] << 16); r[2 * e + 1] -= __uint_as_float(h[e] & 0xffff0000u); }
        }
        o[p] = make_uint4(h[0], h[1], h[2], h[3]);
    }
}
// eight e4m3 times a power of two as bf16
__device__ __forceinline__ uint4 dequant8(uint32_t a, uint32_t b, float sc) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sc, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sc, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sc, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sc, true)));
}

// what a lane's packed row is and sees: keys [0, lim8) in 8 bits, [h0, lim) in bf16
struct Kv8Row {
    int row, head, lim8, h0, lim;     // row < 0: no such row
};
__device__ __forceinline__ Kv8Row kv8_row(const Kv8Attn &a, int b, int kvh, int m) {
    Kv8Row r{-1, kvh * a.G, 0, 0, 0};
    const int i = m / opaque_s(a.G), row = a.s.cu[b] + i;
    if (row >= a.s.cu[b + 1]) return r;
    r.row = row; r.head = kvh * a.G + m - i * a.G;
    const int st = a.s.start[b], n = a.s.count[b];
    if (n == 0) return r;
    r.lim = a.limits ? min(max(a.limits[row], 0), st + n) : st + i + 1;
    const int own = r.lim > 0 ? (r.lim - 1) / KV8_PAGE : 0;
    const bool warm = own >= st / KV8_PAGE;          // older pages are complete and in 8 bits only
    r.h0 = warm ? own * KV8_PAGE : r.lim;
    r.lim8 = r.h0;
    return r;
}

// The sequence of a workgroup.  Workgroups that share a compute unit slow each other, and those of the longest sequences end last: they
// start first, one to a unit (8 sequences of 618 to 2925 tokens in no order, 17 rows of heads 32 / 4 of 128: 25 -> 22 us;
// 12 of 500 to 6000, 32 rows of 32 / 8 in float32 79 -> 70; 8 prompts of 300 behind 300 to 3000 105 -> 92; equal lengths as before).
__device__ __forceinline__ int kv8_sequence(const Kv8Attn &a) {
    return a.order ? (int)min((unsigned)a.order[blockIdx.z], gridDim.z - 1) : (int)blockIdx.z;
}

template <int HD, int SRC>
struct Kv8Planes { static constexpr int N = SRC == KV8_F32 ? 3 : SRC == KV8_FRAG2 ? 2 : 1; };

// q elements e0 .. e0 + 7 of a lane's row, as planes
template <int HD, int SRC>
__device__ __forceinline__ void kv8_q8(const Kv8Attn &a, const Kv8Row &r, int b, int e0, uint4 (&o)[Kv8Planes<HD, SRC>::N]) {
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (SRC == KV8_BF16) {
        o[0] = r.row < 0 ? zero : *(const uint4 *)((const uint16_t *)a.q + (size_t)r.row * a.q_stride + r.head * HD + e0);
    } else if constexpr (SRC == KV8_F32) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r.row >= 0) {
            const float4 *p = (const float4 *)((const float *)a.q + (size_t)r.row * a.q_stride + r.head * HD + e0);
            const float4 x = p[0], y = p[1];
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        }
        split_planes<3>(v, o);
    } else {
        const int ar = r.row < 0 ? 0 : (a.q_row0 ? a.q_row0[b] : 32 * b) + r.row - a.s.cu[b];
        const size_t vec = ((size_t)((ar >> 5) * a.Hq + r.head) * (HD / 16)) * 64 + frag_vec(ar & 31, e0 >> 3);
        o[0] = r.row < 0 ? zero : a.qhi[vec];
        if constexpr (SRC == KV8_FRAG2) o[1] = r.row < 0 ? zero : a.qlo[vec];
    }
}
// Q fragments of a tile: [plane][k-step]
template <int HD, int SRC>
__device__ __forceinline__ void kv8_load_q(const Kv8Attn &a, const Kv8Row &r, int b, int half, uint4 (&q)[Kv8Planes<HD, SRC>::N][HD / 16]) {
    constexpr int KSQ = HD / 16;
#pragma unroll
    for (int s = 0; s < KSQ; ++s) {
        uint4 o[Kv8Planes<HD, SRC>::N];
        kv8_q8<HD, SRC>(a, r, b, 16 * s + 8 * half, o);
#pragma unroll
        for (int p = 0; p < Kv8Planes<HD, SRC>::N; ++p) q[p][s] = o[p];
    }
}

// The reference of a step over 64 keys (raw scores of two tiles of 32 keys; the lane's keys are key0 + r and key0 + 32 + r), by which
// sum and result are rescaled: the largest score when it was last moved.  It moves where a score is more than
// 2^8 weights above it, not with every new maximum (of 32 rows one has a new maximum on almost every page of the first few thousand
// keys): weights are then at most 2^8, as exact relative to each other as before.
constexpr float KV8_SLACK = 8.f;      // log2 of the largest weight
// the larger of three (a NaN is passed over, as by fmaxf, whose operands are first made canonical: twice the instructions)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
template <bool MASK, int HT>
__device__ __forceinline__ void kv8_rescale(f32x16 (&sacc)[2], int key0, int hi, float scale_log2e, float &m_run, float &l_run, f32x16 (&oacc)[HT]) {
    if (MASK) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (key0 + r >= hi) sacc[0][r] = -INFINITY;
            if (key0 + 32 + r >= hi) sacc[1][r] = -INFINITY;
        }
    }
    float m0 = max3(sacc[0][0], sacc[0][1], sacc[0][2]), m1 = max3(sacc[1][0], sacc[1][1], sacc[1][2]);
#pragma unroll
    for (int r = 3; r < 15; r += 2) { m0 = max3(m0, sacc[0][r], sacc[0][r + 1]); m1 = max3(m1, sacc[1][r], sacc[1][r + 1]); }
    const float mx = fmaxf(max3(m0, sacc[0][15], sacc[1][15]), m1);
    if (__builtin_amdgcn_ballot_w64((mx - m_run) * scale_log2e > KV8_SLACK)) {
        const float m_new = fmaxf(m_run, fmaxf(mx, shx(mx, 32)));
        const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * scale_log2e);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int tt = 0; tt < HT; ++tt)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[tt][r] *= alpha;
    }
}
// Registers 8 hh .. + 7 of O^T tile tt of a lane's row, normalised: channels 32 tt + 8 q + 4 half .. + 3, q = 2 hh, 2 hh + 1
template <int HD, int SRC>
__device__ __forceinline__ void kv8_store(const Kv8Attn &a, const Kv8Row &r, int tt, int hh, const float (&o)[8], int lane) {
    const int half = lane >> 5;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int q = 2 * hh + i;
        // (a row that sees nothing is not masked where the others of its tile need no mask)
        const float v0 = r.lim > 0 ? o[4 * i] : 0.f, v1 = r.lim > 0 ? o[4 * i + 1] : 0.f, v2 = r.lim > 0 ? o[4 * i + 2] : 0.f, v3 = r.lim > 0 ? o[4 * i + 3] : 0.f;
        if constexpr (SRC >= KV8_FRAG) {    // the partner lane holds the other half of an octet: see attn_write_frag
            const float w0 = shx(v0, 32), w1 = shx(v1, 32), w2 = shx(v2, 32), w3 = shx(v3, 32);
            if (i == half && r.row >= 0) {
                const float v[8] = {half ? w0 : v0, half ? w1 : v1, half ? w2 : v2, half ? w3 : v3, half ? v0 : w0, half ? v1 : w1, half ? v2 : w2, half ? v3 : w3};
                uint4 hi, lo;
                pack8_split(v, hi, lo);
                const size_t vec = (size_t)(r.row >> 5) * (a.Hq * HD / 16) * 64 + frag_vec(r.row & 31, r.head * (HD / 8) + tt * 4 + q);
                a.xhi[vec] = hi;
                a.xlo[vec] = lo;
            }
        } else if (r.row >= 0) {
            const size_t at = (size_t)r.row * a.out_stride + r.head * HD + 32 * tt + 8 * q + 4 * half;
            if constexpr (SRC == KV8_BF16) *(uint2 *)((uint16_t *)a.out + at) = make_uint2(f2bf2(v0, v1), f2bf2(v2, v3));
            else *(float4 *)((float *)a.out + at) = make_float4(v0, v1, v2, v3);
        }
    }
}

// The NS shares of a tile, in order of range: eight registers of O^T tile tt, normalised.  rl: the lane's row of the tile.
template <int HD>
__device__ __forceinline__ void kv8_sum(const float *p0, int NS, int tt, int hh, int lane, float m_init, float scale_log2e, float (&o)[8]) {
    constexpr int PF = AttnPartial<HD>::FLOATS, CH = 8;       // CH ranges are requested together
    const float *ml = p0 + 32 * HD + 2 * (lane & 31), *po = p0 + ((tt * 4 + 2 * hh) * 64 + lane) * 4;
    float M = m_init, L = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
    for (int s0 = 0; s0 < NS; s0 += CH) {
        float2 x[CH];
        float4 v[CH][2];
#pragma unroll
        for (int u = 0; u < CH; ++u) x[u] = s0 + u < NS ? *(const float2 *)(ml + (size_t)(s0 + u) * PF) : make_float2(m_init, 0.f);
#pragma unroll
        for (int u = 0; u < CH; ++u)
            if (s0 + u < NS)
#pragma unroll
                for (int e = 0; e < 2; ++e) v[u][e] = *(const float4 *)(po + (size_t)(s0 + u) * PF + e * 256);
        float mn = M;
#pragma unroll
        for (int u = 0; u < CH; ++u) mn = fmaxf(mn, x[u].x);
        const float f0 = __builtin_amdgcn_exp2f((M - mn) * scale_log2e);
        M = mn;
        L *= f0;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= f0;
#pragma unroll
        for (int u = 0; u < CH; ++u)
            if (s0 + u < NS) {
                const float f = __builtin_amdgcn_exp2f((x[u].x - M) * scale_log2e);
                L += f * x[u].y;
#pragma unroll
                for (int e = 0; e < 2; ++e) { o[4 * e] += f * v[u][e].x; o[4 * e + 1] += f * v[u][e].y; o[4 * e + 2] += f * v[u][e].z; o[4 * e + 3] += f * v[u][e].w; }
            }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= inv;
}

// The number of a sequence's page u; -1 for one that is no page's.  It is asked for before the loads of an earlier page and made
// uniform (waited for) behind them: a wait where it is asked for is one for every load of the wave that is on its way.
__device__ __forceinline__ int kv8_ask(const Kv8State &s, const int *table, int u) { return table[min(u, s.max_blocks - 1)]; }
__device__ __forceinline__ int kv8_page(const Kv8State &s, int asked) {
    const int id = __builtin_amdgcn_readfirstlane(asked);
    return (unsigned)id < (unsigned)s.n_pages ? id : -1;
}

// Smallest and largest over the rows of a tile (the lanes of a group of ROWS) of what they see; rows that see nothing count as none.
struct Kv8Span { int min8, max8, hmin, hmax; };     // 8-bit keys all rows see / some row sees; hot pages [hmin, hmax]
template <int ROWS>
__device__ __forceinline__ Kv8Span kv8_span(const Kv8Row &r) {
    const bool sees = r.lim > 0, warm = sees && r.h0 < r.lim;
    Kv8Span s{sees ? r.lim8 : 0x7fffffff, r.lim8, warm ? r.h0 / KV8_PAGE : 0x7fffffff, warm ? r.h0 / KV8_PAGE : -1};
#pragma unroll
    for (int off = 1; off < ROWS; off <<= 1) {
        s.min8 = min(s.min8, shx(s.min8, off)); s.max8 = max(s.max8, shx(s.max8, off));
        s.hmin = min(s.hmin, shx(s.hmin, off)); s.hmax = max(s.hmax, shx(s.hmax, off));
    }
    s.min8 = __builtin_amdgcn_readfirstlane(s.min8); s.max8 = __builtin_amdgcn_readfirstlane(s.max8);
    s.hmin = __builtin_amdgcn_readfirstlane(s.hmin); s.hmax = __builtin_amdgcn_readfirstlane(s.hmax);
    return s;
}

// Few packed rows (decoding): a tile of 16 per workgroup, whose four waves share the pages of a key range; a wave streams its pages
// straight to registers.  The products are 16 x 16 x 32: one token of a group of four fills a quarter of the operand's rows, of
// 32 x 32 x 16 an eighth, and O, Q and the scores take half the registers, so that no wave keeps any in memory, where each
// reload would wait for all pages that are on their way.  The launch is a chain of latencies where contexts are short: a wave
// asks for its first page before it knows what its rows see.  Where they are long it is a stream of memory: each wave has half a page or
// more (8 KB with head_dim 128) on its way, K of the next page during the softmax, V during the next scores.
// The waves' results meet in LDS and, with several key ranges, in memory, where the last workgroup to arrive adds them up.
// Operands (lane: n = lane % 16, g = lane / 16): a K operand's row 4 a + i is key 8 a + 4 kb + i of 32, so that a lane of S^T holds
// keys 8 g .. + 7 of each tile of 32, which is the P operand's order; a lane's eight bytes are half of a chunk's sixteen.
// STREAM: the sequence has no other tile (launches of several tiles read a page once per tile, from L2).
// grid: x = kv head + Hkv * key range, y tile, z sequence; 256 threads
typedef __attribute__((ext_vector_type(4))) float f32x4;
__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// eight bytes that nobody else of this launch reads: not to be kept in L2
__device__ __forceinline__ uint2 load8_stream(const uint8_t *p) {
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
    const u32x2 x = __builtin_nontemporal_load((const u32x2 *)p);
    return make_uint2(x.x, x.y);
}
template <int HD>
struct Kv8Part16 { static constexpr int FLOATS = 16 * HD + 32; };   // per (tile of 16, kv head, range): O [HD/16][64 lanes][4], (M, L)[16]

// its workgroups that a compute unit holds
template <int HD, int SRC>
constexpr int kv8_few_resident() { return HD == 128 && (SRC == KV8_F32 || SRC == KV8_FRAG2) ? 2 : 3; }

template <int HD, int SRC, bool STREAM>
__global__ __launch_bounds__(256, (kv8_few_resident<HD, SRC>())) void k_kv8_attn_few(const Kv8Attn a) {
    constexpr int T = HD / 32, CB = HD / 16, N = Kv8Planes<HD, SRC>::N, PF = Kv8Part16<HD>::FLOATS;   // T: k-steps of 32, and chunks per 32 keys
    constexpr int W = 4, NB = (CB + W - 1) / W;        // waves; channel blocks that a wave adds up
    __shared__ float4 s_o[4][CB][64];
    __shared__ float s_ml[W][2][16];
    __shared__ int s_flag;
    const int tidx = opaque_tid();
    const int w = __builtin_amdgcn_readfirstlane(tidx >> 6), lane = tidx & 63, n = lane & 15, g = lane >> 4;
    const int b = kv8_sequence(a), rt = blockIdx.y, kvh = blockIdx.x % opaque_s(a.Hkv), split = blockIdx.x / opaque_s(a.Hkv);
    const int stride = W * a.NS;
    const int *table = a.s.table + (size_t)b * a.s.max_blocks;
    int u = split * W + w;
    const int ask0 = kv8_ask(a.s, table, u);
    int ask = kv8_ask(a.s, table, u + stride);
    // a lane's place in a chunk: storage row of its key (kb = 0; kb = 1: 8 rows on), half and octet of the elements
    const int krow = (n & 3) + 4 * (n >> 3) + 8 * ((n >> 1) & 2);
    const int k_off = ((g & 1) * 32 + krow) * 16 + 8 * (g >> 1), v_off = ((g >> 1) * 32 + n) * 16 + 8 * (g & 1);
    uint2 kc[2][2][T], vc[2][CB];
    float ks1, vs1;
    auto get = [](const uint8_t *p) { return STREAM ? load8_stream(p) : *(const uint2 *)p; };
    auto load_k = [&](int id) {
        const size_t at = (size_t)max(id, 0) * a.Hkv + kvh;      // (a page that does not exist is read as page 0 and masked)
        const uint8_t *p = a.pages + at * (2 * KV8_PAGE * HD) + k_off;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) kc[j][kb][t] = get(p + (j * T + t) * 1024 + kb * 128);
        ks1 = a.scales[at * 2];
    };
    auto load_v = [&](int id) {
        const size_t at = (size_t)max(id, 0) * a.Hkv + kvh;
        const uint8_t *p = a.pages + at * (2 * KV8_PAGE * HD) + KV8_PAGE * HD + v_off;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int c = 0; c < CB; ++c) vc[j][c] = get(p + (j * T + (c >> 1)) * 1024 + (c & 1) * 256);
        vs1 = a.scales[at * 2 + 1];
    };
    int id = kv8_page(a.s, ask0);
    if (rt * 16 >= (a.s.cu[b + 1] - a.s.cu[b]) * a.G) return;
    load_k(id);
    const Kv8Row r = kv8_row(a, b, kvh, rt * 16 + n);
    uint4 q[N][T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        uint4 o[N];
        kv8_q8<HD, SRC>(a, r, b, 32 * t + 16 * (g >> 1) + 8 * (g & 1), o);
#pragma unroll
        for (int p = 0; p < N; ++p) q[p][t] = o[p];
    }
    load_v(id);
    const Kv8Span sp = kv8_span<16>(r);
    const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
    f32x4 oacc[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) oacc[c] = zero4;
    float m_run = a.m_init, l_run = 0.f;
    // scores of 64 keys to weights and result: kf(tile, kb, step), vf(tile, channel block): fragments in bf16
    auto scores = [&](f32x4 (&s)[2][2], auto kf) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                s[j][kb] = zero4;
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const uint4 k = kf(j, kb, t);
#pragma unroll
                    for (int p = 0; p < N; ++p) s[j][kb] = mfma16(k, q[p][t], s[j][kb]);
                }
            }
    };
    auto softmax = [&](auto masked, f32x4 (&s)[2][2], int page, int hi) {
        if (decltype(masked)::value) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (page * KV8_PAGE + 32 * j + 8 * g + 4 * kb + i >= hi) s[j][kb][i] = -INFINITY;
        }
        auto at = [&](int e) { return s[e >> 3][(e >> 2) & 1][e & 3]; };
        float mx = max3(at(0), at(1), at(2)), m1 = max3(at(3), at(4), at(5));
#pragma unroll
        for (int e = 6; e < 14; e += 4) { mx = max3(mx, at(e), at(e + 1)); m1 = max3(m1, at(e + 2), at(e + 3)); }
        mx = fmaxf(max3(mx, at(14), at(15)), m1);
        if (__builtin_amdgcn_ballot_w64((mx - m_run) * a.scale_log2e > KV8_SLACK)) {     // (see kv8_rescale)
            mx = fmaxf(mx, shx(mx, 16));
            const float m_new = fmaxf(m_run, fmaxf(mx, shx(mx, 32)));
            const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * a.scale_log2e);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int c = 0; c < CB; ++c) oacc[c] *= alpha;
        }
        const float mb = m_run * a.scale_log2e;
        float ls = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[e >> 3][(e >> 2) & 1][e & 3], a.scale_log2e, -mb));
            s[e >> 3][(e >> 2) & 1][e & 3] = x;
            ls += x;
        }
        l_run += ls;
    };
    auto values = [&](const f32x4 (&s)[2][2], auto vf) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float pr[8] = {s[j][0][0], s[j][0][1], s[j][0][2], s[j][0][3], s[j][1][0], s[j][1][1], s[j][1][2], s[j][1][3]};
            uint4 ph[N];
            split_planes<N>(pr, ph);
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const uint4 v = vf(j, c);
#pragma unroll
                for (int p = 0; p < N; ++p) oacc[c] = mfma16(v, ph[p], oacc[c]);
            }
        }
    };
    const int n8 = (sp.max8 + KV8_PAGE - 1) / KV8_PAGE, nh = max(0, sp.hmax - sp.hmin + 1);
    f32x4 s[2][2];
    auto page_step = [&](auto masked) {
        const int ask2 = kv8_ask(a.s, table, u + 2 * stride);
        const float ks = ks1, vs = vs1;
        scores(s, [&](int j, int kb, int t) { return dequant8(kc[j][kb][t].x, kc[j][kb][t].y, ks); });
        const int id1 = kv8_page(a.s, ask);
        if (u + stride < n8) load_k(id1);
        softmax(masked, s, u, id >= 0 ? r.lim8 : 0);
        values(s, [&](int j, int c) { return dequant8(vc[j][c].x, vc[j][c].y, vs); });
        if (u + stride < n8) load_v(id1);
        id = id1; ask = ask2;
        u += stride;
    };
    // (pages that all rows see whole, if they see anything, need no mask: see k_kv8_attn_many)
    while (u < n8 && (u + 1) * KV8_PAGE <= sp.min8 && id >= 0) page_step(std::false_type{});
    while (u < n8) page_step(std::true_type{});
    for (; u < n8 + nh; u += stride) {       // hot pages
        const int page = sp.hmin + u - n8;
        const size_t off = (size_t)b * a.hot.seq_stride + (size_t)kvh * a.hot.head_stride + (size_t)((page * KV8_PAGE + a.s.hotbase[b]) & a.hot.mask) * HD;
        const uint4 *kp = (const uint4 *)(a.hot.k + off) + (g & 1) * 32 + krow, *vp = (const uint4 *)(a.hot.v + off) + (g >> 1) * 32 + n;
        scores(s, [&](int j, int kb, int t) { return kp[(j * CB + 2 * t + (g >> 1)) * 64 + 8 * kb]; });
        softmax(std::true_type{}, s, page, r.h0 < r.lim && r.h0 / KV8_PAGE == page ? r.lim : 0);
        values(s, [&](int j, int c) { return vp[(j * CB + (c >> 1) * 2 + (g & 1)) * 64 + (c & 1) * 16]; });
    }
    // the waves' shares meet: every wave adds up a part of the channels
    l_run += shx(l_run, 16);
    l_run += shx(l_run, 32);
    if (lane < 16) { s_ml[w][0][lane] = m_run; s_ml[w][1][lane] = l_run; }
    __syncthreads();
    float M = a.m_init, L = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) M = fmaxf(M, s_ml[i][0][n]);
#pragma unroll
    for (int i = 0; i < W; ++i) L += s_ml[i][1][n] * __builtin_amdgcn_exp2f((s_ml[i][0][n] - M) * a.scale_log2e);
    const float f = __builtin_amdgcn_exp2f((m_run - M) * a.scale_log2e);
    auto scaled = [&](int c) { return make_float4(oacc[c][0] * f, oacc[c][1] * f, oacc[c][2] * f, oacc[c][3] * f); };
#pragma unroll
    for (int c = 0; c < CB; ++c) s_o[w][c][lane] = scaled(c);
    __syncthreads();
    float o[NB][4];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        const int cb = min(w + k * W, CB - 1);
        const float4 x0 = s_o[0][cb][lane], x1 = s_o[1][cb][lane], x2 = s_o[2][cb][lane], x3 = s_o[3][cb][lane];
        o[k][0] = (x0.x + x1.x) + (x2.x + x3.x); o[k][1] = (x0.y + x1.y) + (x2.y + x3.y);
        o[k][2] = (x0.z + x1.z) + (x2.z + x3.z); o[k][3] = (x0.w + x1.w) + (x2.w + x3.w);
    }
    if (a.NS > 1) {
        const size_t item = (size_t)(b * a.rts + rt) * a.Hkv + kvh;
        float *p0 = a.part + item * a.NS * PF, *pp = p0 + (size_t)split * PF;
#pragma unroll
        for (int k = 0; k < NB; ++k)
            if (w + k * W < CB && r.row >= 0) store16_agent(pp + ((w + k * W) * 64 + lane) * 4, o[k][0], o[k][1], o[k][2], o[k][3]);
        if (w == 0 && lane < 16 && r.row >= 0) st_agent2(pp + 16 * HD + 2 * lane, M, L);
        if (!arrive_last(a.counters + item, a.NS, &s_flag)) return;
        constexpr int CH = 8 / NB;       // ranges requested together
        M = a.m_init; L = 0.f;
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[k][e] = 0.f;
        if (r.row >= 0)
            for (int s0 = 0; s0 < a.NS; s0 += CH) {
                float2 x[CH], v[CH][NB][2];
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const float *ps = p0 + (size_t)min(s0 + i, a.NS - 1) * PF;
                    x[i] = ld_agent2(ps + 16 * HD + 2 * n);
#pragma unroll
                    for (int k = 0; k < NB; ++k) {
                        const float *po = ps + (min(w + k * W, CB - 1) * 64 + lane) * 4;
                        v[i][k][0] = ld_agent2(po);
                        v[i][k][1] = ld_agent2(po + 2);
                    }
                }
                float mn = M;
#pragma unroll
                for (int i = 0; i < CH; ++i) mn = fmaxf(mn, x[i].x);
                const float f0 = __builtin_amdgcn_exp2f((M - mn) * a.scale_log2e);
                M = mn;
                L *= f0;
#pragma unroll
                for (int k = 0; k < NB; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[k][e] *= f0;
#pragma unroll
                for (int i = 0; i < CH; ++i)
                    if (s0 + i < a.NS) {
                        const float fi = __builtin_amdgcn_exp2f((x[i].x - M) * a.scale_log2e);
                        L += fi * x[i].y;
#pragma unroll
                        for (int k = 0; k < NB; ++k) { o[k][0] += fi * v[i][k][0].x; o[k][1] += fi * v[i][k][0].y; o[k][2] += fi * v[i][k][1].x; o[k][3] += fi * v[i][k][1].y; }
                    }
            }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        if (w + k * W >= CB) break;
        // (a row that sees nothing is not masked where the others of its tile need no mask)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][e] = r.lim > 0 ? o[k][e] * inv : 0.f;
        const int ch = (w + k * W) * 16 + 4 * g;
        if constexpr (SRC >= KV8_FRAG) {     // lanes 16 apart hold the two halves of an octet: one writes its high plane, one its low
            const float x0 = shx(o[k][0], 16), x1 = shx(o[k][1], 16), x2 = shx(o[k][2], 16), x3 = shx(o[k][3], 16);
            const bool odd = g & 1;
            const float v8[8] = {odd ? x0 : o[k][0], odd ? x1 : o[k][1], odd ? x2 : o[k][2], odd ? x3 : o[k][3], odd ? o[k][0] : x0, odd ? o[k][1] : x1, odd ? o[k][2] : x2, odd ? o[k][3] : x3};
            uint4 hi, lo;
            pack8_split(v8, hi, lo);
            if (r.row >= 0) {
                const size_t vec = (size_t)(r.row >> 5) * (a.Hq * HD / 16) * 64 + frag_vec(r.row & 31, r.head * (HD / 8) + (ch >> 3));
                if (odd) a.xlo[vec] = lo; else a.xhi[vec] = hi;
            }
        } else if (r.row >= 0) {
            const size_t at = (size_t)r.row * a.out_stride + r.head * HD + ch;
            if constexpr (SRC == KV8_BF16) *(uint2 *)((uint16_t *)a.out + at) = make_uint2(f2bf2(o[k][0], o[k][1]), f2bf2(o[k][2], o[k][3]));
            else *(float4 *)((float *)a.out + at) = make_float4(o[k][0], o[k][1], o[k][2], o[k][3]);
        }
    }
}

// Many packed rows (blocks of a group, prompts): four tiles of 32 per workgroup, one per wave; a page is made bf16 once by all four, in
// LDS.  A step multiplies Q with the keys of page u + 1 under the softmax of page u, whose matrix and vector work do not wait for each
// other, then adds page u's values: K is staged two pages ahead and V one (two waves stage K, two V; from memory to registers one
// more page ahead), with one barrier per page.  grid: x = kv head + Hkv * key range, y group of four tiles counted from the last
// (prompts: the longest start first), z sequence; 256 threads
template <int HD, int SRC>
__global__ __launch_bounds__(256, HD == 128 && SRC == KV8_F32 ? 1 : 2) void k_kv8_attn_many(const Kv8Attn a) {
    constexpr int KSQ = HD / 16, HT = HD / 32, N = Kv8Planes<HD, SRC>::N, FR = HD / 8;    // FR fragments of 1 KB of K, and of V, per page
    constexpr int LPW = HD / 32;           // chunks per wave and page; of the HD / 8 chunks the first half is K
    __shared__ __attribute__((aligned(16))) uint4 buf[2][2][FR * 64];      // [K, V][page mod 2]
    __shared__ int s_span[4][4];
    const int tidx = opaque_tid();
    const int w = __builtin_amdgcn_readfirstlane(tidx >> 6), lane = tidx & 63, half = lane >> 5;
    const int b = kv8_sequence(a), rt0 = (gridDim.y - 1 - blockIdx.y) * 4, kvh = blockIdx.x % opaque_s(a.Hkv), split = blockIdx.x / opaque_s(a.Hkv);
    const int packed = (a.s.cu[b + 1] - a.s.cu[b]) * a.G;
    if (rt0 * 32 >= packed) return;
    const int rt = rt0 + w;
    const bool active = rt * 32 < packed;
    const Kv8Row r = kv8_row(a, b, kvh, rt * 32 + (lane & 31));
    const Kv8Span sp = kv8_span<32>(r);
    if (lane == 0) { s_span[w][0] = sp.max8; s_span[w][1] = sp.hmin; s_span[w][2] = sp.hmax; }
    __syncthreads();
    int max8 = 0, hmin = 0x7fffffff, hmax = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) { max8 = max(max8, s_span[i][0]); hmin = min(hmin, s_span[i][1]); hmax = max(hmax, s_span[i][2]); }
    max8 = __builtin_amdgcn_readfirstlane(max8); hmin = __builtin_amdgcn_readfirstlane(hmin); hmax = __builtin_amdgcn_readfirstlane(hmax);
    uint4 q[N][KSQ];
    kv8_load_q<HD, SRC>(a, r, b, half, q);
    f32x16 oacc[HT];
#pragma unroll
    for (int tt = 0; tt < HT; ++tt)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[tt][e] = 0.f;
    float m_run = a.m_init, l_run = 0.f;
    const int n8 = (max8 + KV8_PAGE - 1) / KV8_PAGE, nh = max(0, hmax - hmin + 1), n = n8 + nh;
    const int per = (n + a.NS - 1) / opaque_s(a.NS), u0 = split * per, u1 = min(n, u0 + per);
    const int *table = a.s.table + (size_t)b * a.s.max_blocks;
    int ask = kv8_ask(a.s, table, u0);
    // Pages that all rows of the wave see whole (those that see anything) need no mask, and take a loop of their own: a mask on a
    // branch costs copies of all scores on the other.  A page that does not exist (read as page 0) needs one.
    bool gone = false;
    for (int i = u0 + lane; i < min(n8, u1); i += 64) gone = gone || (unsigned)table[i] >= (unsigned)a.s.n_pages;
    const int clear = __builtin_amdgcn_ballot_w64(gone) ? u0 : min(min(n8, u1), sp.min8 / KV8_PAGE);
    // what a wave holds of the page on its way: 8-bit chunks with their scale.  (A hot page, of which a workgroup has one or two, is
    // read when it is placed: registers for its fragments on their way would be missing in the products.)
    uint4 raw[LPW];
    float raw_scale = 1.f;
    const bool is_v = w >= 2;
    auto fetch = [&](int u) {
        if (u >= n8) return;
        const int id = kv8_page(a.s, ask);
        ask = kv8_ask(a.s, table, u + 1);
        const size_t at = (size_t)max(id, 0) * a.Hkv + kvh;      // (a page that does not exist is read as page 0 and masked)
        const uint4 *p = (const uint4 *)(a.pages + at * (2 * KV8_PAGE * HD)) + w * LPW * 64 + lane;
#pragma unroll
        for (int c = 0; c < LPW; ++c) raw[c] = p[c * 64];
        raw_scale = a.scales[at * 2 + is_v];
    };
    auto place = [&](int u) {
        uint4 *d = buf[is_v][u & 1] + (w & 1) * 2 * LPW * 64 + lane;
        if (u < n8) {
#pragma unroll
            for (int c = 0; c < LPW; ++c) {
                d[2 * c * 64] = dequant8(raw[c].x, raw[c].y, raw_scale);
                d[(2 * c + 1) * 64] = dequant8(raw[c].z, raw[c].w, raw_scale);
            }
        } else {
            const size_t off = (size_t)b * a.hot.seq_stride + (size_t)kvh * a.hot.head_stride + (size_t)(((hmin + u - n8) * KV8_PAGE + a.s.hotbase[b]) & a.hot.mask) * HD;
            const uint4 *p = (const uint4 *)((is_v ? a.hot.v : a.hot.k) + off) + (w & 1) * 2 * LPW * 64 + lane;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4 x[LPW];
#pragma unroll
                for (int c = 0; c < LPW; ++c) x[c] = p[(h * LPW + c) * 64];
#pragma unroll
                for (int c = 0; c < LPW; ++c) d[(h * LPW + c) * 64] = x[c];
            }
        }
    };
    // Products in groups of two k-steps (four fragments); the next group's fragments are read first and the caller's vector work fills
    // the matrix instructions' time.
    constexpr int GK = KSQ / 2;
    auto scores = [&](f32x16 (&sacc)[2], int u, auto beside) {
        const uint4 *fr = buf[0][u & 1] + lane;
        uint4 k[2][4];
        auto read = [&](int g, uint4 (&d)[4]) { d[0] = fr[2 * g * 64]; d[1] = fr[(KSQ + 2 * g) * 64]; d[2] = fr[(2 * g + 1) * 64]; d[3] = fr[(KSQ + 2 * g + 1) * 64]; };
        read(0, k[0]);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sacc[j][e] = 0.f;
#pragma unroll
        for (int g = 0; g < GK; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            if (g + 1 < GK) read(g + 1, k[(g + 1) & 1]);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int p = 0; p < N; ++p) { sacc[0] = mfma32(k[g & 1][2 * s], q[p][2 * g + s], sacc[0]); sacc[1] = mfma32(k[g & 1][2 * s + 1], q[p][2 * g + s], sacc[1]); }
            beside(g);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const int ahead = is_v ? 1 : 2;      // pages that this wave stages ahead of the one whose values are added
    f32x16 sacc[2];
    if (u0 < u1) {
        fetch(u0);
        place(u0);
        if (u0 + 1 < u1) fetch(u0 + 1);
        if (!is_v && u0 + 1 < u1) { place(u0 + 1); if (u0 + 2 < u1) fetch(u0 + 2); }
        __syncthreads();
        if (active) scores(sacc, u0, [](int) {});
    }
    auto step = [&](auto masked, int u, f32x16 (&sacc)[2], f32x16 (&nacc)[2]) {     // sacc: page u's scores; nacc: the next page's
        __syncthreads();      // page u + 1's keys and page u's values are in LDS; page u's keys and u - 1's values have been read
        if (u + ahead < u1) { place(u + ahead); if (u + ahead + 1 < u1) fetch(u + ahead + 1); }
        if (!active) return;
        constexpr bool MASK = decltype(masked)::value;
        int page = u, hi = 0;
        if (MASK) {
            const bool cold = u < n8;
            page = cold ? u : hmin + u - n8;
            hi = cold ? ((unsigned)__builtin_amdgcn_readfirstlane(table[u]) < (unsigned)a.s.n_pages ? r.lim8 : 0) : (r.h0 < r.lim && r.h0 / KV8_PAGE == page ? r.lim : 0);
        }
        kv8_rescale<MASK, HT>(sacc, page * KV8_PAGE + 16 * half, hi, a.scale_log2e, m_run, l_run, oacc);
        __builtin_amdgcn_s_setprio(1);      // (the other workgroup's wave does its vector work meanwhile: 200 -> 190 us for a prompt of 4096)
        const float mb = m_run * a.scale_log2e;
        float ls[2] = {0.f, 0.f};
        scores(nacc, min(u + 1, u1 - 1), [&](int g) {       // the weights of page u, a share beside every group
#pragma unroll
            for (int e = 16 / GK * g; e < 16 / GK * (g + 1); ++e)
#pragma unroll
                for (int j = 0; j < 2; ++j) { sacc[j][e] = __builtin_amdgcn_exp2f(fmaf(sacc[j][e], a.scale_log2e, -mb)); ls[j] += sacc[j][e]; }
        });
        __builtin_amdgcn_s_setprio(0);
        l_run += ls[0] + ls[1];
        const uint4 *fr = buf[1][u & 1] + lane;
        uint4 v[2][HT];
        auto read = [&](int g, uint4 (&d)[HT]) {       // g = 2 * tile + step
#pragma unroll
            for (int tt = 0; tt < HT; ++tt) d[tt] = fr[((g >> 1) * KSQ + tt * 2 + (g & 1)) * 64];
        };
        read(0, v[0]);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            if (g < 3) read(g + 1, v[(g + 1) & 1]);
            float pr[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) pr[e] = sacc[g >> 1][8 * (g & 1) + e];
            uint4 ph[N];
            split_planes<N>(pr, ph);
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int tt = 0; tt < HT; ++tt) oacc[tt] = mfma32(v[g & 1][tt], ph[p], oacc[tt]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    f32x16 nacc[2];
    int u = u0;
    for (; u + 1 < clear; u += 2) {
        step(std::false_type{}, u, sacc, nacc);
        step(std::false_type{}, u + 1, nacc, sacc);
    }
    for (; u < u1; u += 2) {
        step(std::true_type{}, u, sacc, nacc);
        if (u + 1 < u1) step(std::true_type{}, u + 1, nacc, sacc);
    }
    if (!active) return;
    const float l_tot = l_run + shx(l_run, 32), inv = a.NS > 1 ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
    float *pp = a.part + (((size_t)(b * a.rts + rt) * a.Hkv + kvh) * a.NS + split) * AttnPartial<HD>::FLOATS;
    if (a.NS > 1 && lane < 32) *(float2 *)(pp + 32 * HD + 2 * lane) = make_float2(m_run, l_tot);
#pragma unroll
    for (int tt = 0; tt < HT; ++tt)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = oacc[tt][8 * hh + e] * inv;
            if (a.NS == 1) kv8_store<HD, SRC>(a, r, tt, hh, o, lane);
            else
#pragma unroll
                for (int q = 0; q < 2; ++q) *(float4 *)(pp + ((tt * 4 + 2 * hh + q) * 64 + lane) * 4) = make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
        }
}

// The key ranges of k_kv8_attn_many's tiles meet, one wave per eight registers of an O^T tile (in the launch itself the last workgroup
// to arrive would read all of four tiles' shares alone: 44 us for 8 heads, 32 rows and 16 ranges, 15 + 4 so).
// grid: x kv head, y tile, z sequence; 64 * HD / 16 threads
template <int HD, int SRC>
__global__ __launch_bounds__(512) void k_kv8_merge(const Kv8Attn a) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, b = blockIdx.z, rt = blockIdx.y, kvh = blockIdx.x;
    if (rt * 32 >= (a.s.cu[b + 1] - a.s.cu[b]) * a.G) return;
    const Kv8Row r = kv8_row(a, b, kvh, rt * 32 + (lane & 31));
    float o[8];
    kv8_sum<HD>(a.part + (size_t)((b * a.rts + rt) * a.Hkv + kvh) * a.NS * AttnPartial<HD>::FLOATS, a.NS, w >> 1, w & 1, lane, a.m_init, a.scale_log2e, o);
    kv8_store<HD, SRC>(a, r, w >> 1, w & 1, o, lane);
}

}  // namespace deer
