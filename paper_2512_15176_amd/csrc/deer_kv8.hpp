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
__device__ __forceinline__ int kv8_scan(int v, int *tmp) {   // inclusive sum over 1024 threads; tmp: 16 words of LDS
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __builtin_amdgcn_ds_bpermute((lane - off) << 2, v);
        if (lane >= off) v += o;
    }
    if (lane == 63) tmp[w] = v;
    __syncthreads();
    int base = 0;
    for (int i = 0; i < w; ++i) base += tmp[i];
    __syncthreads();
    return v + base;
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
    for (size_t j = i; j < (size_t)s.max_batch; j += n) { s.len[j] = s.held[j] = s.hot[j] = s.base[j] = s.start[j] = s.count[j] = s.hotbase[j] = s.carry[j] = 0; }
    for (size_t j = i; j <= (size_t)s.max_batch; j += n) s.cu[j] = 0;
    for (size_t j = i; j < (size_t)s.max_rows; j += n) { s.slot[j] = -1; s.row_seq[j] = -1; s.row_pos[j] = 0; }
    if (i < 8) s.stat[i] = i == 0 ? s.n_pages : 0;
}

// Sequence b keeps its first start tokens and takes count rows behind them; afterwards it holds ceil((start + count) / 64) pages.
// Pages given back go on the stack before any is taken from it, such that releases followed by the same requests give the same
// table: taken page i is the i-th page given back (in order of sequence and block), then the stack's top and down.
// A sequence is refused (keeps its pages and tokens, gets no rows) for numbers out of range, a start behind its tokens, a start
// inside a page whose bf16 rows are gone, or, like every growing one behind it, where the pages do not suffice.
// Every workgroup works out all sequences (a few microseconds of scans, once for the launch) and writes its share of table entries
// and rows; the state itself is written by the last to arrive, when all have read it.  grid: any; 1024 threads; B <= 1024.
__global__ __launch_bounds__(1024) void k_kv8_reserve(Kv8State s, const int *__restrict__ start, int start_add, const int *__restrict__ count,
                                                      int count_const, int B, int rows, int max_new, int max_len, int scratch) {
    __shared__ int s_row[KV8_MAX_BATCH], s_start[KV8_MAX_BATCH], s_n[KV8_MAX_BATCH], s_held[KV8_MAX_BATCH], s_tp[KV8_MAX_BATCH],
        s_grow[KV8_MAX_BATCH], s_give[KV8_MAX_BATCH], tmp[16], s_taken, s_refused, s_flag;
    const int b = threadIdx.x;
    int st = 0, n = 0, len = 0, held = 0, hot = 0, base = 0;
    if (b < B) {
        st = (start ? start[b] : 0) + start_add;
        n = count ? count[b] : count_const;
        len = s.len[b]; held = s.held[b]; hot = s.hot[b]; base = s.base[b];
    }
    const int top = s.stat[0];
    if (b == 0) { s_taken = 0; s_refused = 0; }
    const int rn = min(max(n, 0), rows);              // the rows' layout follows the request, granted or not
    const int row_end = kv8_scan(b < B ? rn : 0, tmp), row0 = row_end - (b < B ? rn : 0);
    const bool in_ring = st / KV8_PAGE >= hot, kept = st / KV8_PAGE == base / KV8_PAGE && st <= base;
    bool ok = b < B && st >= 0 && n >= 0 && n <= max_new && st <= max_len && st + n <= max_len && st <= len &&
              ((st & (KV8_PAGE - 1)) == 0 || in_ring || kept) && row_end <= rows;
    const int tp = ok ? (st + n + KV8_PAGE - 1) / KV8_PAGE : held;
    const int grow = max(0, tp - held), give = max(0, held - tp);
    const int grow_end = kv8_scan(grow, tmp), give_end = kv8_scan(give, tmp);
    if (b < KV8_MAX_BATCH) { s_give[b] = give_end; s_grow[b] = grow_end; }
    __syncthreads();
    const int given = s_give[KV8_MAX_BATCH - 1], avail = top + given;
    if (grow > 0 && grow_end > avail) ok = false;
    const int m = ok ? n : 0, first = st / KV8_PAGE, last = (st + max(m, 1) - 1) / KV8_PAGE;
    const int touched = m > 0 ? last - first + 1 : 0;
    const int touched_end = kv8_scan(touched, tmp);
    s_row[b] = b < B ? row0 : 0x7fffffff; s_start[b] = st; s_n[b] = m; s_held[b] = held; s_tp[b] = tp;
    if (ok && grow > 0) atomicMax(&s_taken, grow_end);
    if (b < B && !ok) atomicAdd(&s_refused, 1);
    __syncthreads();
    const int taken = s_taken;
    auto back = [&](int i) {      // the i-th page given back
        const int q = kv8_upper(s_give, KV8_MAX_BATCH, i), off = i - (q ? s_give[q - 1] : 0);
        return s.table[(size_t)q * s.max_blocks + s_tp[q] + off];
    };
    auto take = [&](int i) { return i < given ? back(i) : s.free[top - 1 - (i - given)]; };
    const int tid = blockIdx.x * 1024 + threadIdx.x, nth = gridDim.x * 1024;
    for (int i = tid; i < taken; i += nth) {
        const int q = kv8_upper(s_grow, KV8_MAX_BATCH, i);
        s.table[(size_t)q * s.max_blocks + s_held[q] + i - (q ? s_grow[q - 1] : 0)] = take(i);
    }
    for (int r = tid; r < rows; r += nth) {
        const int q = kv8_upper(s_row, B, r) - 1;
        int sl = -1, sq = -1, ps = 0;
        if (q >= 0 && r - s_row[q] < s_n[q]) {
            ps = s_start[q] + r - s_row[q]; sq = q;
            const int pi = ps / KV8_PAGE;
            const int page = pi < s_held[q] ? s.table[(size_t)q * s.max_blocks + pi] : take((q ? s_grow[q - 1] : 0) + pi - s_held[q]);
            sl = page * KV8_PAGE + ps % KV8_PAGE;
        }
        s.slot[r] = sl; s.row_seq[r] = sq; s.row_pos[r] = ps;
    }
    for (int j = tid; j < given - taken; j += nth) s.free[top + j] = back(given - 1 - j);   // entries from `top` on: read by nobody here
    if (!arrive_last(&s.stat[2], gridDim.x, &s_flag)) return;
    if (b < B) {
        s.start[b] = st; s.count[b] = m; s.cu[b] = min(row0, rows);
        s.hotbase[b] = scratch ? (touched_end - touched - first) * KV8_PAGE : 0;
        if (b == B - 1) s.cu[B] = min(row_end, rows);
        const int older = m > 0 && st % KV8_PAGE ? (in_ring ? 1 : 2) : 0;
        s.carry[b] = scratch || older == 2 ? older : 0;       // (a short pass finds the ring's rows where they are)
        if (ok) {
            s.len[b] = st + n; s.held[b] = tp;
            // (without rows, back inside the kept page: the ring does not hold it)
            s.hot[b] = n > 0 ? max(min(hot, first), last - 1) : st % KV8_PAGE && !in_ring ? hot : min(hot, first);
            s.base[b] = (scratch && older) || (kept && st % KV8_PAGE) ? st : st < base ? first * KV8_PAGE : base;
        }
    }
    for (int i = b; i < given; i += 1024) {
        const int q = kv8_upper(s_give, KV8_MAX_BATCH, i);
        s.table[(size_t)q * s.max_blocks + s_tp[q] + i - (q ? s_give[q - 1] : 0)] = -1;
    }
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
// A page's 64 rows of one head in registers, K and V in fragment order: thread t has the lanes' vectors of chunks t, t + 256, .. (two
// fragments each).  They are quantised into the pool; 256 threads, all of which call it.
template <int HD>
struct Kv8Regs {
    static constexpr int NC = KV8_PAGE * HD / 16;   // chunk lanes of K, and of V
    static constexpr int PER = (NC + 255) / 256;
    uint4 x[2][PER][2];
};
template <int HD>
__device__ __forceinline__ void kv8_quantise(const Kv8Regs<HD> &p, uint8_t *__restrict__ pp, float *__restrict__ scales, float (&s_max)[2][4]) {
    using R = Kv8Regs<HD>;
    float amax[2] = {0.f, 0.f};
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
        for (int i = 0; i < R::PER; ++i) {
            if (R::NC % 256 && threadIdx.x + 256 * i >= R::NC) continue;
            amax[kv] = amax8(amax8(amax[kv], p.x[kv][i][0]), p.x[kv][i][1]);
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) amax[kv] = fmaxf(amax[kv], shx(amax[kv], off));
        if ((threadIdx.x & 63) == 0) s_max[kv][threadIdx.x >> 6] = amax[kv];
    }
    __syncthreads();
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        const float sc = kv8_scale(fmaxf(fmaxf(s_max[kv][0], s_max[kv][1]), fmaxf(s_max[kv][2], s_max[kv][3])));
        const float inv = __uint_as_float((254u << 23) - __float_as_uint(sc));    // 1 / 2^e
        if (threadIdx.x == 0) scales[kv] = sc;
#pragma unroll
        for (int i = 0; i < R::PER; ++i) {
            const int c = threadIdx.x + 256 * i;
            if (R::NC % 256 && c >= R::NC) continue;
            const uint2 a = quant8(p.x[kv][i][0], inv), d = quant8(p.x[kv][i][1], inv);
            *(uint4 *)(pp + (size_t)kv * KV8_PAGE * HD + (size_t)c * 16) = make_uint4(a.x, a.y, d.x, d.y);
        }
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
// grid: x page of the sequence's pass, y kv head, z sequence; 256 threads
template <int HD, typename SrcT>
__global__ __launch_bounds__(256) void k_kv8_append(Kv8State s, const SrcT *__restrict__ k, const SrcT *__restrict__ v, size_t k_stride, size_t v_stride,
                                                    Kv8Hot hot, Kv8Hot ring, int is_long, uint8_t *__restrict__ pages, float *__restrict__ scales, int Hkv) {
    using R = Kv8Regs<HD>;
    constexpr int OCTS = HD / 8, VS = HD + 8;       // padded row of V in LDS
    __shared__ __attribute__((aligned(16))) uint16_t s_v[KV8_PAGE * VS];
    __shared__ int s_bad[KV8_PAGE];
    __shared__ float s_max[2][4];
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
    for (int i = threadIdx.x; i < KV8_PAGE; i += 256) s_bad[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < KV8_PAGE * OCTS; i += 256) {
        const int tok = i / OCTS, oct = i % OCTS;
        if (tok < t0 || tok >= t1) continue;
        const uint4 x = load8_bf16(v + (size_t)(row0 + tok) * v_stride + (size_t)head * HD + oct * 8);
        if (nonfinite8(x)) s_bad[tok] = 1;
        *(uint4 *)(s_v + tok * VS + oct * 8) = x;
    }
    R p;
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
        const int c = threadIdx.x + 256 * i, lane = c & 63, rr = lane & 31;
        if (R::NC % 256 && c >= R::NC) continue;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int f = (c >> 6) * 2 + u, tok = f / (HD / 16) * 32 + 16 * ((rr >> 2) & 1) + 4 * (rr >> 3) + (rr & 3), oct = f % (HD / 16) * 2 + (lane >> 5);
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (tok >= t0 && tok < t1) {
                x = load8_bf16(k + (size_t)(row0 + tok) * k_stride + (size_t)head * HD + oct * 8);
                if (nonfinite8(x)) s_bad[tok] = 1;
            } else if (tok < t0 && (whole || carry)) x = *(const uint4 *)(ring.k + older + ((size_t)f * 64 + lane) * 8);
            p.x[0][i][u] = x;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
        const int c = threadIdx.x + 256 * i, lane = c & 63, rr = lane & 31, half = lane >> 5;
        if (R::NC % 256 && c >= R::NC) continue;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int f = (c >> 6) * 2 + u, blk = f / (HD / 16) * 32;
            const size_t off = ((size_t)f * 64 + lane) * 8;
            {
                const int tok = blk + 16 * ((rr >> 2) & 1) + 4 * (rr >> 3) + (rr & 3);
                const bool mine = tok >= t0 && tok < t1;
                if (mine && s_bad[tok]) p.x[0][i][u] = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
                if (mine || (tok < t0 && carry)) *(uint4 *)(hot.k + at.hot + off) = p.x[0][i][u];
                if (out && (mine || (tok < t0 && carry))) *(uint4 *)(ring.k + at.ring + off) = p.x[0][i][u];
            }
            const int tok0 = blk + 16 * half + 8 * (f & 1), ch = f % (HD / 16) / 2 * 32 + rr;     // eight tokens of a channel
            const bool some = tok0 < t1 && tok0 + 8 > t0, old = tok0 < t0;
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (old && (some || whole || carry)) x = *(const uint4 *)(ring.v + older + off);
            if (some) {
                uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int tok = tok0 + e;
                    const uint32_t y = tok >= t0 && tok < t1 && !s_bad[tok] ? s_v[tok * VS + ch] : tok < t0 ? (w[e >> 1] >> (16 * (e & 1))) & 0xffffu : 0u;
                    w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | y << 16 : (w[e >> 1] & 0xffff0000u) | y;
                }
                x = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if (some || (old && carry)) {
                *(uint4 *)(hot.v + at.hot + off) = x;
                if (out) *(uint4 *)(ring.v + at.ring + off) = x;
            }
            p.x[1][i][u] = x;
        }
    }
    if (!whole) return;      // (the whole workgroup)
    const int id = s.table[(size_t)b * s.max_blocks + page];
    if ((unsigned)id >= (unsigned)s.n_pages) return;
    const size_t pg = (size_t)id * Hkv + head;
    kv8_quantise<HD>(p, pages + pg * (2 * KV8_PAGE * HD), scales + pg * 2, s_max);
}

// Where another kernel has put the pass's rows into the hot pages (the engine's QKV projection): pages that they complete go to the pool,
// and with the rows in the scratch (is_long) the last two pages to the ring.  grid as above
template <int HD>
__global__ __launch_bounds__(256) void k_kv8_settle(Kv8State s, Kv8Hot hot, Kv8Hot ring, int is_long, uint8_t *__restrict__ pages, float *__restrict__ scales, int Hkv) {
    using R = Kv8Regs<HD>;
    __shared__ float s_max[2][4];
    const int b = blockIdx.z, head = blockIdx.y, n = s.count[b];
    if (n == 0) return;
    const int st = s.start[b], end = st + n, first = st / KV8_PAGE, last = (end - 1) / KV8_PAGE, page = first + blockIdx.x;
    if (page > last) return;
    const bool whole = end >= (page + 1) * KV8_PAGE, out = is_long && page >= last - 1;
    if (!whole && !out) return;
    const Kv8At at = kv8_at(s, hot, ring, b, head, page, HD);
    R p;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int i = 0; i < R::PER; ++i) {
            const int c = threadIdx.x + 256 * i;
            if (R::NC % 256 && c >= R::NC) continue;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const size_t off = ((size_t)((c >> 6) * 2 + u) * 64 + (c & 63)) * 8;
                p.x[kv][i][u] = *(const uint4 *)((kv ? hot.v : hot.k) + at.hot + off);
                if (out) *(uint4 *)((kv ? ring.v : ring.k) + at.ring + off) = p.x[kv][i][u];
            }
        }
    if (!whole) return;
    const int id = s.table[(size_t)b * s.max_blocks + page];
    if ((unsigned)id >= (unsigned)s.n_pages) return;
    const size_t pg = (size_t)id * Hkv + head;
    kv8_quantise<HD>(p, pages + pg * (2 * KV8_PAGE * HD), scales + pg * 2, s_max);
}

// Rows as they stand in the cache (complete pages in 8 bits, else bf16) for n (sequence, position) pairs; zeros for a pair that names no
// token.  One thread per (row, octet) of a head: the bytes of 16 tokens of a channel are one 16-byte vector, so that the tokens of a
// workgroup, which mostly follow each other, find theirs in the lines that the first has fetched.  grid: x rows, y head
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
//   less than the result's own rounding), three for float32 (24 bits), two for the engine's fragments (its Q has two planes).
// ------------------------------------------------------------------------------------------
enum { KV8_BF16 = 0, KV8_F32 = 1, KV8_FRAG = 2 };   // where q comes from and the result goes: rows, or the engine's fragments

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
    int Hq, Hkv, G, rows, NS, rts;                 // NS key ranges; rts: tiles of 32 packed rows per sequence
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

template <int HD, int SRC>
struct Kv8Planes { static constexpr int N = SRC == KV8_BF16 ? 1 : SRC == KV8_F32 ? 3 : 2; };

// Q fragments of a tile: [plane][k-step]
template <int HD, int SRC>
__device__ __forceinline__ void kv8_load_q(const Kv8Attn &a, const Kv8Row &r, int b, int half, uint4 (&q)[Kv8Planes<HD, SRC>::N][HD / 16]) {
    constexpr int KSQ = HD / 16;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int s = 0; s < KSQ; ++s) {
        if constexpr (SRC == KV8_BF16) {
            q[0][s] = r.row < 0 ? zero : *(const uint4 *)((const uint16_t *)a.q + (size_t)r.row * a.q_stride + r.head * HD + 16 * s + 8 * half);
        } else if constexpr (SRC == KV8_F32) {
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (r.row >= 0) {
                const float4 *p = (const float4 *)((const float *)a.q + (size_t)r.row * a.q_stride + r.head * HD + 16 * s + 8 * half);
                const float4 x = p[0], y = p[1];
                v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
            }
            uint4 pl[3];
            split_planes<3>(v, pl);
            q[0][s] = pl[0]; q[1][s] = pl[1]; q[2][s] = pl[2];
        } else {
            const int ar = r.row < 0 ? 0 : (a.q_row0 ? a.q_row0[b] : 32 * b) + r.row - a.s.cu[b];
            const size_t vec = ((size_t)((ar >> 5) * a.Hq + r.head) * KSQ + s) * 64 + half * 32 + (ar & 31);
            q[0][s] = r.row < 0 ? zero : a.qhi[vec];
            q[1][s] = r.row < 0 ? zero : a.qlo[vec];
        }
    }
}

// One step over 64 keys: scores (raw, of two tiles of 32 keys; the lane's keys are key0 + r and key0 + 32 + r) to weights, running
// maximum and sum, rescaled result.
template <int HT>
__device__ __forceinline__ void kv8_softmax(f32x16 (&sacc)[2], bool mask, int key0, int lo, int hi, float scale_log2e, float &m_run,
                                            float &l_run, f32x16 (&oacc)[HT]) {
    if (mask) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (key0 + r >= hi || key0 + r < lo) sacc[0][r] = -INFINITY;
            if (key0 + 32 + r >= hi || key0 + 32 + r < lo) sacc[1][r] = -INFINITY;
        }
    }
    float mx = fmaxf(sacc[0][0], sacc[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, fmaxf(sacc[0][r], sacc[1][r]));
    mx = fmaxf(mx, shx(mx, 32));
    const float m_new = fmaxf(m_run, mx);
    const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * scale_log2e);
    const float mb = m_new * scale_log2e;
    float ls0 = 0.f, ls1 = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        sacc[0][r] = __builtin_amdgcn_exp2f(sacc[0][r] * scale_log2e - mb); ls0 += sacc[0][r];
        sacc[1][r] = __builtin_amdgcn_exp2f(sacc[1][r] * scale_log2e - mb); ls1 += sacc[1][r];
    }
    l_run = l_run * alpha + (ls0 + ls1);
    m_run = m_new;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {
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
        const float v0 = o[4 * i], v1 = o[4 * i + 1], v2 = o[4 * i + 2], v3 = o[4 * i + 3];
        if constexpr (SRC == KV8_FRAG) {    // the partner lane holds the other half of an octet: see attn_write_frag
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

// A tile's share of one key range, un-normalised, in register order (see AttnPartial): eight registers of O^T tile tt.  (Agent scope:
// another XCD may read it in this launch.)
template <int HD>
__device__ __forceinline__ void kv8_put(float *pp, int tt, int hh, const float (&o)[8], int lane) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
        store16_agent(pp + ((tt * 4 + 2 * hh + q) * 64 + lane) * 4, o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
}
// The NS shares of a tile, in order of range: eight registers of O^T tile tt, normalised.  rl: the lane's row of the tile.
template <int HD, bool AGENT>
__device__ __forceinline__ void kv8_sum(const float *p0, int NS, int tt, int hh, int lane, float m_init, float scale_log2e, float (&o)[8]) {
    constexpr int PF = AttnPartial<HD>::FLOATS, CH = 8;       // CH ranges are requested together
    const float *ml = p0 + 32 * HD + 2 * (lane & 31), *po = p0 + ((tt * 4 + 2 * hh) * 64 + lane) * 4;
    auto get = [](const float *p) { return AGENT ? ld_agent2(p) : *(const float2 *)p; };
    float M = m_init, L = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
    for (int s0 = 0; s0 < NS; s0 += CH) {
        float2 x[CH], v[CH][4];
#pragma unroll
        for (int u = 0; u < CH; ++u) x[u] = s0 + u < NS ? get(ml + (size_t)(s0 + u) * PF) : make_float2(m_init, 0.f);
#pragma unroll
        for (int u = 0; u < CH; ++u)
            if (s0 + u < NS)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u][e] = get(po + (size_t)(s0 + u) * PF + (e >> 1) * 256 + 2 * (e & 1));
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
                for (int e = 0; e < 4; ++e) { o[2 * e] += f * v[u][e].x; o[2 * e + 1] += f * v[u][e].y; }
            }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= inv;
}

// Smallest and largest over the 32 rows of a tile of what they see; rows that see nothing count as none.
struct Kv8Span { int min8, max8, hmin, hmax; };     // 8-bit keys all rows see / some row sees; hot pages [hmin, hmax]
__device__ __forceinline__ Kv8Span kv8_span(const Kv8Row &r) {
    const bool sees = r.lim > 0, warm = sees && r.h0 < r.lim;
    Kv8Span s{sees ? r.lim8 : 0x7fffffff, r.lim8, warm ? r.h0 / KV8_PAGE : 0x7fffffff, warm ? r.h0 / KV8_PAGE : -1};
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        s.min8 = min(s.min8, shx(s.min8, off)); s.max8 = max(s.max8, shx(s.max8, off));
        s.hmin = min(s.hmin, shx(s.hmin, off)); s.hmax = max(s.hmax, shx(s.hmax, off));
    }
    s.min8 = __builtin_amdgcn_readfirstlane(s.min8); s.max8 = __builtin_amdgcn_readfirstlane(s.max8);
    s.hmin = __builtin_amdgcn_readfirstlane(s.hmin); s.hmax = __builtin_amdgcn_readfirstlane(s.hmax);
    return s;
}

// Few packed rows (decoding): one tile of 32 per workgroup, whose eight waves share the pages of a key range; a wave streams its pages
// straight to registers.  The launch is a chain of latencies where contexts are short, so a wave asks for its first page's number
// before it knows what its rows see, and for the page before it has asked for Q; and a stream of memory where they are long: each
// wave has half a page or more (8 KB with head_dim 128) on its way, K of the next page during the softmax, V during the next products.
// The waves' results meet in LDS and, with several key ranges, in memory, where the last workgroup to arrive adds them up.
// grid: x = kv head + Hkv * key range, y tile, z sequence; 512 threads
template <int HD, int SRC>
__global__ __launch_bounds__(512, 1) void k_kv8_attn_few(const Kv8Attn a) {
    constexpr int KSQ = HD / 16, HT = HD / 32, N = Kv8Planes<HD, SRC>::N, KC = HD / 32, W = 8;   // KC chunks per 32 keys of K, and of V
    __shared__ float s_o[4][HT * 16][64];
    __shared__ float s_ml[W][2][32];
    __shared__ int s_flag;
    const int tidx = opaque_tid();
    const int w = __builtin_amdgcn_readfirstlane(tidx >> 6), lane = tidx & 63, half = lane >> 5;
    const int b = blockIdx.z, rt = blockIdx.y, kvh = blockIdx.x % opaque_s(a.Hkv), split = blockIdx.x / opaque_s(a.Hkv);
    const int stride = W * a.NS, *table = a.s.table + (size_t)b * a.s.max_blocks;
    int u = split * W + w;
    auto page_of = [&](int i) { return __builtin_amdgcn_readfirstlane(table[min(i, a.s.max_blocks - 1)]); };
    auto valid = [&](int id) { return (unsigned)id < (unsigned)a.s.n_pages; };
    auto base_of = [&](int i) { return (size_t)(valid(i) ? i : 0) * a.Hkv + kvh; };   // (a page that does not exist is read as page 0 and masked)
    uint4 kc[2 * KC], vc[2 * KC];
    float ks1, vs1;
    auto load_k = [&](int i) {
        const uint4 *p = (const uint4 *)(a.pages + base_of(i) * (2 * KV8_PAGE * HD)) + lane;
#pragma unroll
        for (int c = 0; c < 2 * KC; ++c) kc[c] = p[c * 64];
        ks1 = a.scales[base_of(i) * 2];
    };
    auto load_v = [&](int i) {
        const uint4 *p = (const uint4 *)(a.pages + base_of(i) * (2 * KV8_PAGE * HD) + KV8_PAGE * HD) + lane;
#pragma unroll
        for (int c = 0; c < 2 * KC; ++c) vc[c] = p[c * 64];
        vs1 = a.scales[base_of(i) * 2 + 1];
    };
    int id = page_of(u), id1 = page_of(u + stride);
    if (rt * 32 >= (a.s.cu[b + 1] - a.s.cu[b]) * a.G) return;
    load_k(id);
    const Kv8Row r = kv8_row(a, b, kvh, rt * 32 + (lane & 31));
    uint4 q[N][KSQ];
    kv8_load_q<HD, SRC>(a, r, b, half, q);
    load_v(id);
    const Kv8Span sp = kv8_span(r);
    f32x16 oacc[HT];
#pragma unroll
    for (int tt = 0; tt < HT; ++tt)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[tt][e] = 0.f;
    float m_run = a.m_init, l_run = 0.f;
    auto scores = [&](f32x16 (&sacc)[2], auto frag) {     // frag(tile, k-step): a K fragment in bf16
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sacc[j][e] = 0.f;
#pragma unroll
        for (int s = 0; s < KSQ; ++s) {
            const uint4 k0 = frag(0, s), k1 = frag(1, s);
#pragma unroll
            for (int p = 0; p < N; ++p) { sacc[0] = mfma32(k0, q[p][s], sacc[0]); sacc[1] = mfma32(k1, q[p][s], sacc[1]); }
        }
    };
    auto values = [&](const f32x16 (&sacc)[2], auto frag) {   // frag(tile, channel tile, step): a V^T fragment
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float pr[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) pr[e] = sacc[j][e];
            uint4 ph[2][N];
            split_planes<N>(pr, ph[0]);
            split_planes<N>(pr + 8, ph[1]);
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int tt = 0; tt < HT; ++tt) {
                    const uint4 v = frag(j, tt, s2);
#pragma unroll
                    for (int p = 0; p < N; ++p) oacc[tt] = mfma32(v, ph[s2][p], oacc[tt]);
                }
        }
    };
    const int n8 = (sp.max8 + KV8_PAGE - 1) / KV8_PAGE, nh = max(0, sp.hmax - sp.hmin + 1);
    for (; u < n8; u += stride) {
        const int id2 = page_of(u + 2 * stride);
        const bool live = valid(id);
        const float ks = ks1, vs = vs1;
        f32x16 sacc[2];
        scores(sacc, [&](int j, int s) {
            const uint4 c = kc[j * KC + (s >> 1)];
            return s & 1 ? dequant8(c.z, c.w, ks) : dequant8(c.x, c.y, ks);
        });
        if (u + stride < n8) load_k(id1);
        const int key0 = u * KV8_PAGE + 16 * half;
        kv8_softmax<HT>(sacc, (u + 1) * KV8_PAGE > sp.min8 || !live, key0, 0, live ? r.lim8 : 0, a.scale_log2e, m_run, l_run, oacc);
        values(sacc, [&](int j, int tt, int s2) {
            const uint4 c = vc[j * KC + tt];
            return s2 ? dequant8(c.z, c.w, vs) : dequant8(c.x, c.y, vs);
        });
        if (u + stride < n8) load_v(id1);
        id = id1; id1 = id2;
    }
    for (; u < n8 + nh; u += stride) {       // hot pages
        const int page = sp.hmin + u - n8;
        const size_t off = (size_t)b * a.hot.seq_stride + (size_t)kvh * a.hot.head_stride + (size_t)((page * KV8_PAGE + a.s.hotbase[b]) & a.hot.mask) * HD;
        const uint4 *kp = (const uint4 *)(a.hot.k + off) + lane, *vp = (const uint4 *)(a.hot.v + off) + lane;
        f32x16 sacc[2];
        scores(sacc, [&](int j, int s) { return kp[(j * KSQ + s) * 64]; });
        const int own = r.h0 < r.lim && r.h0 / KV8_PAGE == page;
        kv8_softmax<HT>(sacc, true, page * KV8_PAGE + 16 * half, 0, own ? r.lim : 0, a.scale_log2e, m_run, l_run, oacc);
        values(sacc, [&](int j, int tt, int s2) { return vp[(j * KSQ + tt * 2 + s2) * 64]; });
    }
    // the waves' shares: waves 4 .. 7 hand theirs to waves 0 .. 3, then every wave adds up eight registers of a tile
    const float l_tot = l_run + shx(l_run, 32);
    if (lane < 32) { s_ml[w][0][lane] = m_run; s_ml[w][1][lane] = l_tot; }
    __syncthreads();
    float M = a.m_init, L = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) M = fmaxf(M, s_ml[i][0][lane & 31]);
#pragma unroll
    for (int i = 0; i < W; ++i) L += s_ml[i][1][lane & 31] * __builtin_amdgcn_exp2f((s_ml[i][0][lane & 31] - M) * a.scale_log2e);
    const float f = __builtin_amdgcn_exp2f((m_run - M) * a.scale_log2e);
    if (w >= 4)
#pragma unroll
        for (int tt = 0; tt < HT; ++tt)
#pragma unroll
            for (int e = 0; e < 16; ++e) s_o[w - 4][tt * 16 + e][lane] = oacc[tt][e] * f;
    __syncthreads();
    if (w < 4)
#pragma unroll
        for (int tt = 0; tt < HT; ++tt)
#pragma unroll
            for (int e = 0; e < 16; ++e) s_o[w][tt * 16 + e][lane] += oacc[tt][e] * f;
    __syncthreads();
    const int tt = w >> 1, hh = w & 1;
    const bool on = tt < HT;
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = min(tt, HT - 1) * 16 + 8 * hh + e;
        o[e] = (s_o[0][i][lane] + s_o[1][i][lane]) + (s_o[2][i][lane] + s_o[3][i][lane]);
    }
    if (a.NS > 1) {
        const size_t item = (size_t)(b * a.rts + rt) * a.Hkv + kvh;
        float *p0 = a.part + item * a.NS * AttnPartial<HD>::FLOATS, *pp = p0 + (size_t)split * AttnPartial<HD>::FLOATS;
        if (on && r.row >= 0) kv8_put<HD>(pp, tt, hh, o, lane);
        if (w == 0 && lane < 32 && r.row >= 0) st_agent2(pp + 32 * HD + 2 * lane, M, L);
        if (!arrive_last(a.counters + item, a.NS, &s_flag) || !on) return;
        if (r.row >= 0) kv8_sum<HD, true>(p0, a.NS, tt, hh, lane, a.m_init, a.scale_log2e, o);
    } else {
        const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= inv;
    }
    if (on) kv8_store<HD, SRC>(a, r, tt, hh, o, lane);
}

// Many packed rows (blocks of a group, prompts): four tiles of 32 per workgroup, one per wave; a page is made bf16 once by all four, in
// LDS, double-buffered with one barrier per page: page i + 1 goes from registers to LDS and page i + 2 from memory to registers
// under the products of page i.  grid: x = kv head + Hkv * key range, y group of four tiles counted from the last (prompts: the
// longest start first), z sequence; 256 threads
template <int HD, int SRC>
__global__ __launch_bounds__(256, HD == 128 && SRC == KV8_F32 ? 1 : 2) void k_kv8_attn_many(const Kv8Attn a) {
    constexpr int KSQ = HD / 16, HT = HD / 32, N = Kv8Planes<HD, SRC>::N, FR = HD / 8;    // FR fragments of 1 KB of K, and of V, per page
    constexpr int LPW = HD / 32;           // chunks per wave and page; of the HD / 8 chunks the first half is K
    __shared__ __attribute__((aligned(16))) uint4 buf[2][2 * FR * 64];
    __shared__ int s_span[4][4];
    const int tidx = opaque_tid();
    const int w = __builtin_amdgcn_readfirstlane(tidx >> 6), lane = tidx & 63, half = lane >> 5;
    const int b = blockIdx.z, rt0 = (gridDim.y - 1 - blockIdx.y) * 4, kvh = blockIdx.x % opaque_s(a.Hkv), split = blockIdx.x / opaque_s(a.Hkv);
    const int packed = (a.s.cu[b + 1] - a.s.cu[b]) * a.G;
    if (rt0 * 32 >= packed) return;
    const int rt = rt0 + w;
    const bool active = rt * 32 < packed;
    const Kv8Row r = kv8_row(a, b, kvh, rt * 32 + (lane & 31));
    const Kv8Span sp = kv8_span(r);
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
    auto valid = [&](int id) { return (unsigned)id < (unsigned)a.s.n_pages; };
    // what a wave holds of the page on its way: 8-bit chunks with their scale, or bf16 fragments
    uint4 raw[2 * LPW];
    float raw_scale = 1.f;
    const bool is_v = w >= 2;
    auto fetch = [&](int u) {
        if (u < n8) {
            const int t = __builtin_amdgcn_readfirstlane(table[u]);
            const size_t at = (size_t)(valid(t) ? t : 0) * a.Hkv + kvh;
            const uint4 *p = (const uint4 *)(a.pages + at * (2 * KV8_PAGE * HD)) + w * LPW * 64 + lane;
#pragma unroll
            for (int c = 0; c < LPW; ++c) raw[c] = p[c * 64];
            raw_scale = a.scales[at * 2 + is_v];
        } else {
            const size_t off = (size_t)b * a.hot.seq_stride + (size_t)kvh * a.hot.head_stride + (size_t)(((hmin + u - n8) * KV8_PAGE + a.s.hotbase[b]) & a.hot.mask) * HD;
            const uint4 *p = (const uint4 *)((is_v ? a.hot.v : a.hot.k) + off) + (w & 1) * 2 * LPW * 64 + lane;
#pragma unroll
            for (int c = 0; c < 2 * LPW; ++c) raw[c] = p[c * 64];
        }
    };
    auto place = [&](int u) {
        uint4 *d = buf[u & 1] + w * 2 * LPW * 64 + lane;
        if (u < n8) {
#pragma unroll
            for (int c = 0; c < LPW; ++c) {
                d[2 * c * 64] = dequant8(raw[c].x, raw[c].y, raw_scale);
                d[(2 * c + 1) * 64] = dequant8(raw[c].z, raw[c].w, raw_scale);
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2 * LPW; ++c) d[c * 64] = raw[c];
        }
    };
    if (u0 < u1) {
        fetch(u0);
        place(u0);
        if (u0 + 1 < u1) fetch(u0 + 1);
    }
    for (int u = u0; u < u1; ++u) {
        __syncthreads();      // page u is in LDS, and page u - 1 has been read by all
        if (u + 1 < u1) { place(u + 1); if (u + 2 < u1) fetch(u + 2); }
        const bool cold = u < n8;
        const int page = cold ? u : hmin + u - n8;
        int lo = 0, hi = cold ? r.lim8 : (r.h0 < r.lim && r.h0 / KV8_PAGE == page ? r.lim : 0);
        if (cold && !valid(__builtin_amdgcn_readfirstlane(table[u]))) hi = 0;
        const bool mask = !cold || (u + 1) * KV8_PAGE > sp.min8 || hi == 0;
        if (!active || (cold && u * KV8_PAGE >= sp.max8) || (!cold && (page < sp.hmin || page > sp.hmax))) continue;
        const uint4 *fr = buf[u & 1] + lane;
        f32x16 sacc[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sacc[j][e] = 0.f;
#pragma unroll
        for (int s = 0; s < KSQ; ++s) {
            const uint4 k0 = fr[s * 64], k1 = fr[(KSQ + s) * 64];
#pragma unroll
            for (int p = 0; p < N; ++p) { sacc[0] = mfma32(k0, q[p][s], sacc[0]); sacc[1] = mfma32(k1, q[p][s], sacc[1]); }
        }
        kv8_softmax<HT>(sacc, __builtin_amdgcn_ballot_w64(mask) != 0, page * KV8_PAGE + 16 * half, lo, hi, a.scale_log2e, m_run, l_run, oacc);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float pr[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) pr[e] = sacc[j][e];
            uint4 ph[2][N];
            split_planes<N>(pr, ph[0]);
            split_planes<N>(pr + 8, ph[1]);
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int tt = 0; tt < HT; ++tt) {
                    const uint4 v = fr[(FR + j * KSQ + tt * 2 + s2) * 64];
#pragma unroll
                    for (int p = 0; p < N; ++p) oacc[tt] = mfma32(v, ph[s2][p], oacc[tt]);
                }
        }
    }
    if (!active) return;
    const float l_tot = l_run + shx(l_run, 32), inv = a.NS > 1 ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
    float *pp = a.part + ((size_t)((b * a.rts + rt) * a.Hkv + kvh) * a.NS + split) * AttnPartial<HD>::FLOATS;
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
    kv8_sum<HD, false>(a.part + (size_t)((b * a.rts + rt) * a.Hkv + kvh) * a.NS * AttnPartial<HD>::FLOATS, a.NS, w >> 1, w & 1, lane, a.m_init, a.scale_log2e, o);
    kv8_store<HD, SRC>(a, r, w >> 1, w & 1, o, lane);
}

}  // namespace deer
