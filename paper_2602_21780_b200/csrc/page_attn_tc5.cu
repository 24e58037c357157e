// Attention of many query rows a head over the 4-bit or 8-bit pages, on the 5th-generation tensor cores (tcgen05.mma,
// accumulators in tensor memory): out = softmax(scale q K^T, causal, window) V.
//
// A unit is (sequence, pair of 128-row query tiles, key/value head), a row being (new token, query head of the
// group); its steps are the pages that its rows see.  A first kernel lists the units' steps (ragged lengths, causal and
// windowed ranges are known on the device only); the attention kernel, one CTA per multiprocessor, deals the steps out
// in contiguous spans weighted by their cost, and a third merges, in a fixed order, units that several CTAs share.
//
// Inside a CTA (16 warps), as in the attention over the contiguous cache:
//   warps 0-3, 4-7 : softmax of query tile A / B, one row a thread, lazily updated maximum;
//   warps 8-13     : producers: code words of a page's record -> fp16 tiles in shared memory, 128-byte-swizzled.  A lane's
//                    words hold 8 consecutive channels of 8 tokens (keys) or 16 tokens of 8 channels (values), so both
//                    tiles are written 16 bytes at a time without exchanging anything, the values transposed
//                    ([channel][token], so that both products read K-major tiles), if the page's tokens stand in the order
//                    position 16 j + 4 m + 2 b + h = token 16 m + 8 b + 2 j + h;
//   warps 14, 15   : one thread each issues S = Q K^T and O += P V (P from tensor memory) of query tile A / B.
// Bound by the softmax warps' exponentials and issue slots next to the tensor pipe (at head_dim 128 both need about
// 1000 clocks a page and tile pair), not by memory: a page is read once per 256 rows.
// Queries are scaled by a power of two per row (largest element in [1, 2)), which the row's logit factor takes back, so
// that bf16 of any size fits; P is fp16, sums and accumulators are float32.  Every wait is bounded; when one runs out the
// kernel runs to its end and the rows it touched become NaN.
//
// Measured.  1374 tokens on 21 984, 16 heads of 64, 4 bit: 217 us, 590 TFLOP/s (0.42 of the sustained bf16 peak; the kernel for few
// rows took 788); 6 chunks of 300 to 2047 tokens on up to 9000, 32 / 8 heads of 128, in bursts: 4 bit 400 us, 872 TFLOP/s (0.61), 8 bit 380 us,
// 917 TFLOP/s (0.65; 373 without the products that bring the values to their unit); call after call, under the power cap, 8 bit takes 395 to
// 413 us (0.60 to 0.62).  At head_dim 64 the exponentials alone, 16 a clock and multiprocessor, take about 115 us of the frame.
// The softmax warps are busy 90 % of the time, the producers wait 55 % of it for free stages.  Storing the tiles
// through generic addresses cost 20 %; the second half of the logits arriving under the first half's exponentials and the
// range of unmasked pages known per unit gave 5 %; a share of 1/8 of the exponentials as polynomials cost 10 %; quarters of the logits with
// the next step's first one ahead cost 4 to 7 % (more waits, more registers).  A unit's begin and end took 17 % of the chunks: queries by
// asynchronous copies under the results' way out, parts in an order that a warp writes whole, 32-bit divisions: 5 to 8 %.
#include <algorithm>

#include "page8_layout.cuh"
#include "page_attn.cuh"
#include "tc5_ptx.cuh"
#include "xsv_kernels.h"

namespace {

constexpr int BM = 128, NPROD = 6, NTHREADS = (8 + NPROD + 2) * 32;
// Cost of a step with two query tiles, with one, and of entering a unit, in ticks: the steps' are the ratios of the attention over the
// contiguous cache; a unit's is fitted, over eight mixes (6 chunks of 300 to 2047 tokens, 40 of 60 to 300, 3 of 400 to 700 on 8000, one of 300 on 60 000, 20
// with a window of 500, a prompt of 2000, 100 prompts of 100 to 400, 8 chunks of 70 to 150 on up to 20 000), heads of 64 and 128, both kinds of pages:
// 100 is 2 to 3 % slower than 144, 160 and 200 at heads of 128, 0.5 % at heads of 64, and these three are within 1.2 % of one another; single mixes differ
// by up to 5 % either way.
constexpr int COST_PAIR = 16, COST_SINGLE = 13, COST_UNIT = 160, MIN_SPAN = 320;
// A row sum that reaches 2^8: look for the maximum again.  Over 8-bit pages weights and sums are 2^P_BIAS larger, still below fp16's largest
// value, so that a weight keeps fp16's full significand down to 2^-21 of the maximum.
constexpr float P_BIAS = 7.f;
template <int BITS> constexpr float SUM_LIMIT = BITS == 8 ? 32768.f : 256.f;
constexpr float NO_MAX = -1e30f;

template <int D> struct Cfg {
    static constexpr int BLK = D / 64;                               // 64-channel blocks of a row
    static constexpr int NBUF = D == 64 ? 3 : 2;                     // S buffers per query tile
    static constexpr int NSTAGE = D == 64 ? 8 : 4;
    static constexpr uint32_t Q_TILE = 128u * 128u * BLK, K_TILE = 64u * 128u * BLK, V_TILE = 128u * D, STAGE = K_TILE + V_TILE;
    static constexpr uint32_t OFF_KV = 2 * Q_TILE, OFF_BAR = OFF_KV + NSTAGE * STAGE, SMEM = OFF_BAR + 1024 + 1024;
    // barriers
    static constexpr int KFULL = 0, VFULL = NSTAGE, EMPTY = 2 * NSTAGE, SFULL = 3 * NSTAGE, PREADY = SFULL + 2 * NBUF,
                         PVDONE = PREADY + 2 * NBUF, QFULL = PVDONE + 2 * NBUF, DRAIN = QFULL + 2, COUNT = DRAIN + 2;
    static_assert(COUNT * 8 + 128 <= 1024 && SMEM <= 227 * 1024, "shared memory");
    __host__ __device__ static constexpr uint32_t tm_s(int x, int b) { return (uint32_t)((x * NBUF + b) * 64); }
    __host__ __device__ static constexpr uint32_t tm_o(int x) { return (uint32_t)(2 * NBUF * 64 + x * D); }
    static_assert(2 * NBUF * 64 + 2 * D <= 512, "tensor memory");
    static constexpr uint32_t IDESC_QK = (1u << 4) | (64u >> 3 << 17) | ((uint32_t)(BM >> 4) << 24);
    static constexpr uint32_t IDESC_PV = (1u << 4) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
    static constexpr int PART = 256 * (D + 2);                       // floats of a part: [D / 4][256 rows] of 4 channels, then (maximum, sum) of the rows
};

// One pair of query tiles of one sequence, for every head alike.
struct alignas(16) Entry {
    int seq, row0, p0, pages;
    int t0, first, n_rows, ticks;     // first new token, its position, query rows of the sequence, cost of one head
};
struct Work {
    int* head;              // [0] entries, [2..3] total ticks of all heads (64-bit)
    int4* desc;             // [CTAs] a unit that begins to be shared: {entry, head, parts, 0}
    long long* pre;         // [entries + 1] ticks before each entry, one head
    Entry* entry;
    float* part;            // [CTAs][2]
    int G, room;            // CTAs; entries that there is room for
};
__device__ __forceinline__ Entry load_entry(const Work& w, int e) {
    Entry n;
    const int4 a = reinterpret_cast<const int4*>(w.entry + e)[0], b = reinterpret_cast<const int4*>(w.entry + e)[1];
    n.seq = a.x; n.row0 = a.y; n.p0 = a.z; n.pages = a.w;
    n.t0 = b.x; n.first = b.y; n.n_rows = b.z; n.ticks = b.w;
    return n;
}

// ------------------------------------------------------------------ the work list
__global__ void __launch_bounds__(1024) page_list_kernel(const __grid_constant__ PageAttn p, const __grid_constant__ Work w) {
    __shared__ int s_base[XSV_PAGE_MAX_SEQS];
    __shared__ long long s_warp[32];
    xsv_dep_release();
    xsv_dep_sync();
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    auto scan = [&](long long v, long long& all) {           // exclusive, over the block
        long long x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) s_warp[wid] = x;
        __syncthreads();
        long long y = s_warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long z = __shfl_up_sync(0xFFFFFFFFu, y, o);
            if (lane >= o) y += z;
        }
        all = __shfl_sync(0xFFFFFFFFu, y, 31);
        const long long before = __shfl_sync(0xFFFFFFFFu, y, (wid + 31) & 31);
        return x - v + (wid ? before : 0);
    };
    auto pairs_of = [&](int s) {
        const int rows = page_seq(p, s).new_ * p.group;
        return rows > p.row_limit ? (rows + 255) / 256 : 0;
    };
    const int per = (p.n_seqs + 1023) / 1024, s0 = min(p.n_seqs, tid * per), s1 = min(p.n_seqs, s0 + per);
    long long n = 0, all;
    for (int s = s0; s < s1; ++s) n += pairs_of(s);
    long long at = scan(n, all);
    for (int s = s0; s < s1; ++s) { s_base[s] = (int)min(at, (long long)w.room); at += pairs_of(s); }
    const int entries = (int)min(all, (long long)w.room);      // all of them, unless the offsets contradict each other
    __syncthreads();
    for (int s = wid; s < p.n_seqs; s += 32) {
        const PageSeq q = page_seq(p, s);
        const int rows = q.new_ * p.group, pairs = rows > p.row_limit ? (rows + 255) / 256 : 0;
        for (int m = lane; m < pairs && s_base[s] + m < entries; m += 32) {
            Entry e;
            e.seq = s; e.row0 = m * 256; e.n_rows = rows; e.first = q.first;
            e.t0 = min(max(p.cu[s], 0), p.n_tokens);
            const int here = min(256, rows - e.row0);
            int lo, hi, h;
            page_row(p, e.row0, lo, h);
            page_row(p, e.row0 + here - 1, hi, h);
            const int last = q.first + hi;                    // position of the last row
            e.p0 = p.window > 0 ? max(0, q.first + lo - p.window + 1) / XSV_PAGE : 0;
            e.pages = max(1, (last < 0 ? 0 : min(last / XSV_PAGE + 1, p.width)) - e.p0);
            e.ticks = COST_UNIT + e.pages * (here > BM ? COST_PAIR : COST_SINGLE);
            int4* dst = reinterpret_cast<int4*>(w.entry + s_base[s] + m);
            dst[0] = make_int4(e.seq, e.row0, e.p0, e.pages);
            dst[1] = make_int4(e.t0, e.first, e.n_rows, e.ticks);
        }
    }
    __syncthreads();
    long long carry = 0;
    for (int base = 0; base < entries; base += 1024) {
        const int e = base + tid;
        const long long t = e < entries ? w.entry[e].ticks : 0, x = scan(t, all);
        if (e < entries) w.pre[e] = carry + x;
        carry += all;
    }
    if (tid == 0) {
        w.pre[entries] = carry;
        w.head[0] = entries;
        *reinterpret_cast<long long*>(w.head + 2) = carry * p.pool.heads;
    }
}

// ------------------------------------------------------------------ the units of a CTA
struct Units {
    int e, h, entries, heads;
    long long base, t0, t1;      // ticks before the unit; the CTA's span
    Entry en;
    int kv0, kv1;                // its steps here
    bool valid;
};
__device__ __forceinline__ int step_cost(const Entry& en) { return en.n_rows - en.row0 > BM ? COST_PAIR : COST_SINGLE; }
__device__ __forceinline__ void settle(const Work& w, Units& u) {          // from the current unit on, one with steps here
    for (;;) {
        if (u.e >= u.entries || u.base >= u.t1) { u.valid = false; return; }
        const int cost = step_cost(u.en);
        // steps that begin before a tick of the unit (a unit's ticks are a 32-bit number; so are its divisions)
        auto steps = [&](long long tick) {
            const long long x = tick - u.base - COST_UNIT;
            return x <= 0 ? 0 : x >= (long long)u.en.pages * cost ? u.en.pages : (int)(((uint32_t)x + cost - 1) / (uint32_t)cost);
        };
        u.kv0 = steps(u.t0);
        u.kv1 = steps(u.t1);
        if (u.kv0 < u.kv1) { u.valid = true; return; }
        u.base += u.en.ticks;
        if (++u.h == u.heads) {
            u.h = 0;
            if (++u.e < u.entries) u.en = load_entry(w, u.e);
        }
    }
}
__device__ __forceinline__ void next_unit(const Work& w, Units& u) {
    u.base += u.en.ticks;
    if (++u.h == u.heads) {
        u.h = 0;
        if (++u.e < u.entries) u.en = load_entry(w, u.e);
    }
    settle(w, u);
}

struct Cta {
    uint8_t* smem;
    uint32_t base, bars, tmem;
    volatile int* abort_flag;
    int* status;
    uint32_t page_ok;            // [stages] ints: whether the stage's page exists
};

// ------------------------------------------------------------------ producers
// Code pairs -> fp16: the magic exponent makes the pair 1024 + code (or, 4 bits up, 64 + code), the subtraction is exact,
// then code * s + z is rounded once.
__device__ __forceinline__ uint32_t dq_lo(uint32_t w, uint32_t s, uint32_t z) { return hfma2_u(hsub2_u((w & 0x000F000Fu) | 0x64006400u, 0x64006400u), s, z); }
__device__ __forceinline__ uint32_t dq_hi(uint32_t w, uint32_t s, uint32_t z) { return hfma2_u(hsub2_u((w & 0x00F000F0u) | 0x54005400u, 0x54005400u), s, z); }
// the row of the key tile, and the column of S and the value tile, of token 16 m + 8 b + 2 j + h
__host__ __device__ constexpr int place(int m, int b, int j, int h) { return 16 * j + 4 * m + 2 * b + h; }
__host__ __device__ constexpr int token_at(int pos) { return 16 * (pos >> 2 & 3) + 8 * (pos >> 1 & 1) + 2 * (pos >> 4) + (pos & 1); }

// A plain load: blocks of this kernel can be resident while the append before it still writes the records, and what
// the wait for it makes visible is not promised to the read-only path.
__device__ __forceinline__ uint4 ld16(const uint8_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void sts16(uint32_t at, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

template <typename T, int D>
__device__ __noinline__ void producer_loop(const PageAttn& p, const Work& w, const Cta c, Units u) {
    using C = Cfg<D>;
    using R = PageRec<D>;
    constexpr int SLABS = 2 * C::BLK;                          // 64 x 64 slabs of a page: keys, then values
    const int lane = threadIdx.x & 31, pw = (threadIdx.x >> 5) - 8, g = lane >> 2, j = lane & 3, odd = g & 1;
    auto BAR = [&](int i) { return c.bars + 8u * (uint32_t)i; };
    struct Regs { uint4 code[4], a[2], b[2]; };                // codes; keys: scale, offset of two 32-channel halves;
                                                               // values: scale, offset rows of tokens 2 j, 2 j + 1
    uint32_t it = 0;                                           // steps of the CTA before the unit
    int slab = pw;                                             // this warp's next slab, counted from the unit's first
    for (; u.valid; next_unit(w, u)) {
        const int n = u.kv1 - u.kv0, total = min(u.en.first + u.en.n_rows / p.group, p.width * XSV_PAGE);
        const int* row = p.table + (size_t)u.en.seq * p.width + u.en.p0 + u.kv0;
        int ids = -1, ids_from = -32;                          // page indices of 32 steps, one a lane
        auto page_of = [&](int k) {
            if (k - ids_from >= 32) {
                ids_from = k & ~31;
                const int pg = u.en.p0 + u.kv0 + ids_from + lane;
                ids = ids_from + lane < n && pg < p.width && pg * XSV_PAGE < total ? row[ids_from + lane] : -1;
                if ((unsigned long long)(long long)ids >= (unsigned long long)p.pool.n_pages) ids = -1;
            }
            return __shfl_sync(0xFFFFFFFFu, ids, k & 31);
        };
        auto fetch = [&](int sl, int page, Regs& r) {
            if (page < 0) return;
            const uint8_t* rec = page_rec<D>(p.pool, page, u.h);
            const int part = sl % SLABS;
            if (part < C::BLK) {
                // 32-channel halves in an order of the lane's own, so that a store's lanes touch different banks
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int kg = 2 * part + (i ^ odd);
                    r.code[2 * i] = ld16(rec + R::K_CODES + (2 * kg * 32 + lane) * 16);
                    r.code[2 * i + 1] = ld16(rec + R::K_CODES + ((2 * kg + 1) * 32 + lane) * 16);
                    r.a[i] = ld16(rec + R::K_SCALE + 64 * kg + 16 * j);
                    r.b[i] = ld16(rec + R::K_ZERO + 64 * kg + 16 * j);
                }
            } else {
                const int v = part - C::BLK;
#pragma unroll
                for (int t = 0; t < 4; ++t) r.code[t] = ld16(rec + R::V_CODES + ((t * C::BLK + v) * 32 + lane) * 16);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    r.a[i] = ld16(rec + R::V_SCALE + 128 * v + 32 * j + 16 * i);
                    r.b[i] = ld16(rec + R::V_ZERO + 128 * v + 32 * j + 16 * i);
                }
            }
        };
        Regs cur{}, nxt{};
        int page = -1, page_n = -1;
        if (slab < n * SLABS) {
            page = page_of(slab / SLABS);
            fetch(slab, page, cur);
        }
        while (slab < n * SLABS) {
            const int k = slab / SLABS, part = slab % SLABS, next = slab + NPROD;
            if (next < n * SLABS) {
                page_n = page_of(next / SLABS);
                fetch(next, page_n, nxt);
            }
            const uint32_t step = it + (uint32_t)k, st = step % C::NSTAGE;
            if (step >= (uint32_t)C::NSTAGE) mbar_wait(BAR(C::EMPTY + (int)st), (step / C::NSTAGE - 1u) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_STAGE);
            const int pg = u.en.p0 + u.kv0 + k, held = total - pg * XSV_PAGE;      // tokens of the page
            const uint32_t stage = c.base + C::OFF_KV + st * C::STAGE;
            if (part < C::BLK) {
                const uint32_t tile = stage + part * 8192;
                if (part == 0 && lane == 0) asm volatile("st.shared.b32 [%0], %1;" ::"r"(c.page_ok + 4u * st), "r"(page >= 0 ? 1 : 0) : "memory");
                if (page >= 0 && held >= XSV_PAGE) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int chunk = 4 * (i ^ odd) + j;
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            const uint32_t w0 = word(cur.code[2 * i], m), w1 = word(cur.code[2 * i + 1], m);
                            const uint4 lo = make_uint4(dq_lo(w0, cur.a[i].x, cur.b[i].x), dq_lo(w0 >> 8, cur.a[i].y, cur.b[i].y),
                                                        dq_lo(w1, cur.a[i].z, cur.b[i].z), dq_lo(w1 >> 8, cur.a[i].w, cur.b[i].w));
                            const uint4 hi = make_uint4(dq_hi(w0, cur.a[i].x, cur.b[i].x), dq_hi(w0 >> 8, cur.a[i].y, cur.b[i].y),
                                                        dq_hi(w1, cur.a[i].z, cur.b[i].z), dq_hi(w1 >> 8, cur.a[i].w, cur.b[i].w));
                            sts16(tile + swz(place(m, 0, g >> 1, odd), chunk), lo);
                            sts16(tile + swz(place(m, 1, g >> 1, odd), chunk), hi);
                        }
                    }
                } else {
                    // the unfilled page's keys as they came; zeros where there is no token or no page
                    const T* tail = tail_rows<T, D>(p.pool, u.en.seq, pg, u.h) + 64 * part + 8 * j;
#pragma unroll 2
                    for (int i = 0; i < 16; ++i) {
                        const int m = i >> 2, b = i >> 1 & 1, half = (i & 1) ^ odd, tok = 16 * m + 8 * b + g;
                        uint4 x = make_uint4(0u, 0u, 0u, 0u);
                        if (page >= 0 && tok < held) x = *reinterpret_cast<const uint4*>(tail + (size_t)tok * D + 32 * half);
                        sts16(tile + swz(place(m, b, g >> 1, odd), 4 * half + j), make_uint4(to_h2<T>(x.x), to_h2<T>(x.y), to_h2<T>(x.z), to_h2<T>(x.w)));
                    }
                }
            } else {
                const int v = part - C::BLK;
                const uint32_t tile = stage + C::K_TILE + v * 8192;
                uint32_t s[8], z[8];                           // tokens 8 i + 2 j, 8 i + 2 j + 1
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[i] = pair_at(cur.a[0], cur.a[1], i);
                    z[i] = pair_at(cur.b[0], cur.b[1], i);
                }
                if (page < 0 || held < XSV_PAGE) {             // places without a token: zeros, whatever the record holds there
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int left = page < 0 ? 0 : held - 8 * i - 2 * j;
                        const uint32_t keep = left >= 2 ? 0xFFFFFFFFu : left == 1 ? 0xFFFFu : 0u;
                        s[i] &= keep;
                        z[i] &= keep;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {                  // channels 8 g + 2 i, 8 g + 2 i + 1
                    uint32_t e[8], o[8];                       // their 16 tokens, in pairs
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint32_t x = word(cur.code[t], i);
                        e[2 * t] = dq_lo(x, s[2 * t], z[2 * t]);
                        o[2 * t] = dq_hi(x, s[2 * t], z[2 * t]);
                        e[2 * t + 1] = dq_lo(x >> 8, s[2 * t + 1], z[2 * t + 1]);
                        o[2 * t + 1] = dq_hi(x >> 8, s[2 * t + 1], z[2 * t + 1]);
                    }
                    const uint4 e0 = make_uint4(e[0], e[1], e[2], e[3]), e1 = make_uint4(e[4], e[5], e[6], e[7]);
                    const uint4 o0 = make_uint4(o[0], o[1], o[2], o[3]), o1 = make_uint4(o[4], o[5], o[6], o[7]);
                    const int re = 8 * g + 2 * i;
                    sts16(tile + swz(re, 2 * j + odd), odd ? e1 : e0);
                    sts16(tile + swz(re, 2 * j + (odd ^ 1)), odd ? e0 : e1);
                    sts16(tile + swz(re + 1, 2 * j + odd), odd ? o1 : o0);
                    sts16(tile + swz(re + 1, 2 * j + (odd ^ 1)), odd ? o0 : o1);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR((part < C::BLK ? C::KFULL : C::VFULL) + (int)st));
            cur = nxt;
            page = page_n;
            slab = next;
        }
        it += (uint32_t)n;
        slab -= n * SLABS;
    }
}

// 8-bit pages: the codes as fp16.  The softmax warps take in the keys' scale, which stands beside a stage's page.  The values' scale 2^ev goes
// into the operand: a unit's output is summed in units of 2^ref, and codes, whole numbers of 2^-9 up to 448, times 2^(ev - ref) are exact in
// fp16 from 2^-15 to 2^7.  So pages whose scales are up to 2^22 apart share a ref, and the weights have nothing to do with scales.  ref is
// settled for 32 steps at a time and changes as little as it can; where the scales of 32 pages are further apart each page is its own ref, and the
// softmax warps move the output when ref changes.  (The exponent in the logits instead, as it once was, cost the weights beside a page with a
// single large value their bits, or all of themselves.)
// A slab is 64 tokens x 64 channels of keys, or half the values: at head_dim 128 all channels of 32 tokens (a lane's 8 tokens are
// 8 consecutive columns of the tile), at 64 all 64 tokens.
template <typename T, int D>
__device__ __noinline__ void producer8_loop(const PageAttn& p, const Work& w, const Cta c, Units u) {
    using C = Cfg<D>;
    using R = Page8Rec<D>;
    constexpr int SLABS = 2 * C::BLK;
    const int lane = threadIdx.x & 31, pw = (threadIdx.x >> 5) - 8, g = lane >> 2, j = lane & 3, odd = g & 1;
    auto BAR = [&](int i) { return c.bars + 8u * (uint32_t)i; };
    constexpr int MOVE_MIN = -15, MOVE_MAX = 7, REF_MIN = P8_EXP_MIN - MOVE_MIN, NO_REF = -1000;
    struct Regs { uint4 code[8]; float scale; };
    struct Step { int page, ref, move; };                      // its page (-1: none), what its output is counted in, and the values' way there
    uint32_t it = 0;                                           // steps of the CTA before the unit
    int slab = pw;                                             // this warp's next slab, counted from the unit's first
    for (; u.valid; next_unit(w, u)) {
        const int n = u.kv1 - u.kv0, total = min(u.en.first + u.en.n_rows / p.group, p.width * XSV_PAGE);
        const int* row = p.table + (size_t)u.en.seq * p.width + u.en.p0 + u.kv0;
        // pages, refs and ev - ref of 32 steps, one a lane; the last ref (a warp looks at every 32 steps that a unit has, in order)
        int ids = -1, refs = 0, moves = 0, ids_from = -32, ref = NO_REF;
        auto step_of = [&](int k) {
            if (k - ids_from >= 32) {
                ids_from = k & ~31;
                const int pg = u.en.p0 + u.kv0 + ids_from + lane;
                ids = ids_from + lane < n && pg < p.width && pg * XSV_PAGE < total ? row[ids_from + lane] : -1;
                if ((unsigned long long)(long long)ids >= (unsigned long long)p.pool.n_pages) ids = -1;
                const bool is = ids >= 0;
                int ev = 0;
                if (is) ev = p8_exponent_of(reinterpret_cast<const float*>(page8_rec<D>(p.pool, ids, u.h) + R::PARAMS)[1]);
                const int hi = __reduce_max_sync(0xFFFFFFFFu, is ? ev : NO_REF), lo = __reduce_min_sync(0xFFFFFFFFu, is ? ev : -NO_REF);
                if (hi - lo <= MOVE_MAX - MOVE_MIN) {          // (no page at all: as before)
                    if (hi >= lo) ref = max(min(max(ref == NO_REF ? (hi + lo) / 2 + 4 : ref, hi - MOVE_MAX), lo - MOVE_MIN), REF_MIN);
                    refs = ref == NO_REF ? 0 : ref;
                } else {
                    refs = max(is ? ev : hi, REF_MIN);
                    ref = __shfl_sync(0xFFFFFFFFu, refs, 31);
                }
                moves = is ? ev - refs : 0;
            }
            return Step{__shfl_sync(0xFFFFFFFFu, ids, k & 31), __shfl_sync(0xFFFFFFFFu, refs, k & 31), __shfl_sync(0xFFFFFFFFu, moves, k & 31)};
        };
        auto fetch = [&](int sl, int page, Regs& r) {
            if (page < 0) return;
            const uint8_t* rec = page8_rec<D>(p.pool, page, u.h);
            const int part = sl % SLABS;
            if (part < C::BLK) {
#pragma unroll
                for (int a = 0; a < 8; ++a) r.code[a] = ld16(rec + R::K_CODES + ((a * C::BLK + part) * 32 + lane) * 16);
                if (part == 0) r.scale = *reinterpret_cast<const float*>(rec + R::PARAMS);
            } else if (D == 128) {
#pragma unroll
                for (int i = 0; i < 8; ++i) r.code[i] = ld16(rec + R::V_CODES + ((8 * (part - C::BLK) + i) * 32 + lane) * 16);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint2 x = *reinterpret_cast<const uint2*>(rec + R::V_CODES + (2 * i * 32 + lane) * 8);
                    const uint2 y = *reinterpret_cast<const uint2*>(rec + R::V_CODES + ((2 * i + 1) * 32 + lane) * 8);
                    r.code[i] = make_uint4(x.x, x.y, y.x, y.y);
                }
            }
        };
        Regs cur{}, nxt{};
        Step here{-1, 0, 0}, ahead{-1, 0, 0};
        if (slab < n * SLABS) {
            here = step_of(slab / SLABS);
            fetch(slab, here.page, cur);
        }
        while (slab < n * SLABS) {
            const int k = slab / SLABS, part = slab % SLABS, next = slab + NPROD;
            if (next < n * SLABS) {
                ahead = step_of(next / SLABS);
                fetch(next, ahead.page, nxt);
            }
            const uint32_t step = it + (uint32_t)k, st = step % C::NSTAGE;
            if (step >= (uint32_t)C::NSTAGE) mbar_wait(BAR(C::EMPTY + (int)st), (step / C::NSTAGE - 1u) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_STAGE);
            const int held = here.page < 0 ? 0 : total - (u.en.p0 + u.kv0 + k) * XSV_PAGE;      // tokens of the page
            const uint32_t stage = c.base + C::OFF_KV + st * C::STAGE;
            if (part < C::BLK) {
                const uint32_t tile = stage + part * 8192;
                if (part == 0 && lane == 0) {
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(c.page_ok + 4u * st), "r"(here.page >= 0 ? 1 : 0) : "memory");
                    // keys' scale, ref
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(c.page_ok + 4u * C::NSTAGE + 8u * st),
                                 "r"(__float_as_int(here.page >= 0 ? cur.scale : 1.f)), "r"(here.ref) : "memory");
                }
                // 16 channels of a token: two chunks of its row (keys of places without a token are masked, whatever they are)
#pragma unroll
                for (int a = 0; a < 8; ++a) {
                    uint32_t h[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) p8_halves(word(cur.code[a], i), h[2 * i], h[2 * i + 1]);
                    const int r = place(a >> 1, a & 1, g >> 1, odd);
                    sts16(tile + swz(r, 2 * j), make_uint4(h[0], h[1], h[2], h[3]));
                    sts16(tile + swz(r, 2 * j + 1), make_uint4(h[4], h[5], h[6], h[7]));
                }
            } else {
                const int v = part - C::BLK;
                const uint32_t tile = stage + C::K_TILE;
                // 2^move, a pair of fp16 (2^-15 is a subnormal one)
                const uint32_t by = (here.move == MOVE_MIN ? 0x0200u : (uint32_t)(here.move + 15) << 10) * 0x10001u;
                auto values = [&](uint32_t codes, uint32_t& lo, uint32_t& hi) {
                    p8_halves(codes, lo, hi);
                    lo = hmul2_u(lo, by);
                    hi = hmul2_u(hi, by);
                };
                if (held < XSV_PAGE) {                         // places without a token: zeros, whatever the record holds there
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (D == 128) {                        // i = 4 (t % 2) + 2 b + h
                            if (16 * (2 * v + (i >> 2)) + 8 * (i >> 1 & 1) + 2 * j + (i & 1) >= held) cur.code[i] = make_uint4(0u, 0u, 0u, 0u);
                        } else {                               // i = 2 t + b, two tokens
                            const int tok = 8 * i + 2 * j;
                            if (tok >= held) cur.code[i].x = cur.code[i].y = 0u;
                            if (tok + 1 >= held) cur.code[i].z = cur.code[i].w = 0u;
                        }
                    }
                }
                if (D == 128) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {              // channels 16 g + 4 i to + 3: pairs of tokens h = 0, 1 of four (t, b)
                        uint32_t e[4][4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t x = word(cur.code[2 * q], i), y = word(cur.code[2 * q + 1], i);
                            values(__byte_perm(x, y, 0x5140), e[0][q], e[1][q]);
                            values(__byte_perm(x, y, 0x7362), e[2][q], e[3][q]);
                        }
#pragma unroll
                        for (int q = 0; q < 4; q += 2) {       // lanes of odd g in another order, so that a store's lanes touch different banks
                            const uint4 a = make_uint4(e[q][0], e[q][1], e[q][2], e[q][3]), b = make_uint4(e[q + 1][0], e[q + 1][1], e[q + 1][2], e[q + 1][3]);
                            const int r = 16 * g + 4 * i + q;
                            sts16(tile + swz(r + odd, 2 * j + v), odd ? b : a);
                            sts16(tile + swz(r + (odd ^ 1), 2 * j + v), odd ? a : b);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {              // channels 8 g + 4 i to + 3, 16 tokens
                        uint32_t e[4][8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const uint32_t x = word(cur.code[q], i), y = word(cur.code[q], i + 2);
                            values(__byte_perm(x, y, 0x5140), e[0][q], e[1][q]);
                            values(__byte_perm(x, y, 0x7362), e[2][q], e[3][q]);
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint4 a = make_uint4(e[q][0], e[q][1], e[q][2], e[q][3]), b = make_uint4(e[q][4], e[q][5], e[q][6], e[q][7]);
                            const int r = 8 * g + 4 * i + q;
                            sts16(tile + swz(r, 2 * j + odd), odd ? b : a);
                            sts16(tile + swz(r, 2 * j + (odd ^ 1)), odd ? a : b);
                        }
                    }
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR((part < C::BLK ? C::KFULL : C::VFULL) + (int)st));
            cur = nxt;
            here = ahead;
            slab = next;
        }
        it += (uint32_t)n;
        slab -= n * SLABS;
    }
}

// ------------------------------------------------------------------ softmax and epilogue
__device__ __forceinline__ void softmax32(const uint32_t (&v)[32], unsigned long long sc2, unsigned long long nm2, unsigned long long& ls2,
                                          uint32_t (&pk)[16]) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float x0, x1;
        f2_unpack(f2_fma(f2_pack(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), sc2, nm2), x0, x1);
        const float p0 = ex2(x0), p1 = ex2(x1);
        ls2 = f2_add(ls2, f2_pack(p0, p1));
        pk[i >> 1] = pack_h2(p0, p1);
    }
}

// A warp's 32 rows of a query tile, of queries and of results, in turns of ROWS rows with 16 bytes a lane, so that global memory
// sees whole rows.  Functions of their own, with their loops rolled: the registers and the instruction cache are the softmax's.
template <int D> struct RowTurns {
    static constexpr int PER_ROW = D / 8, ROWS = 32 / PER_ROW, TURNS = 32 / ROWS;
};
// The rows of a unit on their way into the tile, as they are.  Called when the tile's products with the rows before are done: the
// results' way out hides the latency.
template <typename T, int D>
__device__ __noinline__ void fetch_queries(const PageAttn& p, int t0, int row0, int n_rows, int h, int X, uint32_t tile) {
    constexpr int PER_ROW = RowTurns<D>::PER_ROW, ROWS = RowTurns<D>::ROWS, TURNS = RowTurns<D>::TURNS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, chunk = lane % PER_ROW, first = (warp & 3) * 32 + lane / PER_ROW;
    const T* base = (const T*)p.Q + (size_t)h * p.group * D + 8 * chunk;
    const int q0 = row0 + X * BM;
#pragma unroll 4
    for (int y = 0; y < TURNS; ++y) {
        const int row = first + y * ROWS, q = min(q0 + row, n_rows - 1);
        int qi, qh;
        page_row(p, q, qi, qh);
        cp_async16(tile + (chunk >> 3) * 16384 + swz(row, chunk & 7), base + (size_t)(t0 + qi) * p.q_stride + (size_t)qh * D, q0 + row < n_rows ? 16u : 0u);
    }
    cp_async_commit();
}
// In place: the thread's row -> fp16, its largest element in [1, 2); returns its logit factor.
template <typename T, int D>
__device__ __noinline__ float scale_query(float scale, uint8_t* tile) {
    const int row = threadIdx.x & 127;
    auto at = [&](int k) { return reinterpret_cast<uint4*>(tile + (k >> 3) * 16384 + swz(row, k & 7)); };
    cp_async_wait_all();
    __syncwarp();                                          // the row is other lanes' copies
    float mx = 0.f;
#pragma unroll 4
    for (int k = 0; k < D / 8; ++k) {
        const uint4 x = *at(k);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float2 f = xsv_unpack2<T>(word(x, q));
            mx = fmax3(mx, fabsf(f.x), fabsf(f.y));
        }
    }
    const int e = mx > 0.f ? max((__float_as_int(mx) >> 23) - 127, -126) : 0;
    const float s1 = __int_as_float((127 - e / 2) << 23), s2 = __int_as_float((127 - (e - e / 2)) << 23);
#pragma unroll 1
    for (int k0 = 0; k0 < D / 8; k0 += 4) {
        uint4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = *at(k0 + k);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t z[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float2 f = xsv_unpack2<T>(word(x[k], q));
                z[q] = pack_h2(f.x * s1 * s2, f.y * s1 * s2);
            }
            *at(k0 + k) = make_uint4(z[0], z[1], z[2], z[3]);
        }
    }
    return fmaxf(scale * __int_as_float((127 + min(e, 127)) << 23), MIN_FACTOR);
}

// BITS 8: a page's keys have a scale, which goes into the factor of its logits; its values are counted in 2^ref (see the producers), and so
// is the output, which is brought there when ref changes: exactly, since float32 holds sums of values up to 2^16 in units of the smallest ref,
// 2^-65, and of the smallest values in units of the largest.
template <typename T, int D, int BITS>
__device__ __noinline__ void softmax_loop(const PageAttn& p, const Work& w, const Cta c, Units u) {
    using C = Cfg<D>;
    auto BAR = [&](int i) { return c.bars + 8u * (uint32_t)i; };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, X = warp >> 2, row = tid & 127;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = c.tmem + lane_base + C::tm_s(X, 0), tO = c.tmem + lane_base + C::tm_o(X);
    uint8_t* sQ = c.smem + X * C::Q_TILE;
    auto row_token = [&](int q) { int i, h; page_row(p, q, i, h); return i; };
    uint32_t it = 0, cX = 0;                       // steps of the CTA; steps of this query tile
    bool fetched = false;
    // Completion of the P V of step j (see the attention over the contiguous cache: one barrier per S buffer, never more
    // than one phase ahead of the waits on it)
    auto wait_pv = [&](uint32_t j) { mbar_wait(BAR(C::PVDONE + X * C::NBUF + (int)(j % C::NBUF)), (j / C::NBUF) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_PV); };
    while (u.valid) {
        const int n = u.kv1 - u.kv0, r = u.en.row0 + X * BM + row;
        if (u.en.row0 + X * BM >= u.en.n_rows) {           // no second tile
            it += (uint32_t)n;
            next_unit(w, u);
            continue;
        }
        const int qpos = u.en.first + row_token(min(r, u.en.n_rows - 1)), total = min(u.en.first + u.en.n_rows / p.group, p.width * XSV_PAGE);
        // ---- the query rows (the first unit's are fetched here, the others' ahead)
        if (!fetched) fetch_queries<T, D>(p, u.en.t0, u.en.row0, u.en.n_rows, u.h, X, smem_u32(sQ));
        fetched = false;
        const float sc = scale_query<T, D>(p.scale, sQ);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(C::QFULL + X));

        // pages that every row of the warp sees whole: no mask
        const int q_min = min(__reduce_min_sync(0xFFFFFFFFu, qpos), total - 1), q_max = __reduce_max_sync(0xFFFFFFFFu, qpos);
        const int tok_lo = p.window > 0 ? q_max - p.window + 1 : 0, tok_hi = q_min - (XSV_PAGE - 1);
        float m_used = NO_MAX, l = 0.f;
        int ref_used = 0;
        bool first = true;
        for (int k = 0; k < n; ++k) {
            const int tok0 = (u.en.p0 + u.kv0 + k) * XSV_PAGE;
            const uint32_t buf = cX % C::NBUF, tSb = tS + buf * 64u;
            mbar_wait(BAR(C::SFULL + X * C::NBUF + (int)buf), (cX / C::NBUF) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_S);
            tc_fence_after();
            uint32_t va[32], vb[32], pk[16];
            tmem_ld32(tSb, va);
            int ok;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(ok) : "r"(c.page_ok + 4u * ((it + (uint32_t)k) % C::NSTAGE)) : "memory");
            float sp = sc;
            int ref = 0;
            if (BITS == 8) {
                int ks;
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(ks), "=r"(ref) : "r"(c.page_ok + 4u * C::NSTAGE + 8u * ((it + (uint32_t)k) % C::NSTAGE)) : "memory");
                sp = fmaxf(sc * __int_as_float(ks), MIN_FACTOR);
                if (first) ref_used = ref;
            }
            const bool moved = BITS == 8 && ref != ref_used;           // uniform
            tc_wait_ld();
            tmem_ld32(tSb + 32u, vb);              // arrives under the first half's exponentials
            const bool mask = !(tok0 >= tok_lo && tok0 <= tok_hi && ok);     // uniform
            float ls = 0.f;
            bool careful = first || mask || moved;
            if (!careful) {
                const unsigned long long sc2 = f2_pack(sp, sp), nm2 = f2_pack(BITS == 8 ? P_BIAS - m_used : -m_used, BITS == 8 ? P_BIAS - m_used : -m_used);
                unsigned long long ls2 = f2_pack(0.f, 0.f);
                softmax32(va, sc2, nm2, ls2, pk);
                tmem_st16(tSb, pk);
                tc_wait_ld();
                softmax32(vb, sc2, nm2, ls2, pk);
                tmem_st16(tSb + 16u, pk);
                float l0, l1;
                f2_unpack(ls2, l0, l1);
                ls = l0 + l1;
                careful = __any_sync(0xFFFFFFFFu, !(ls < SUM_LIMIT<BITS>));
            } else {
                tc_wait_ld();
            }
            if (careful) {
                if (mask) {                                // masked places, whatever stands there; visible: lo < token <= hi
                    const int hi = ok ? min(qpos, total - 1) - tok0 : -1, lo = p.window > 0 ? qpos - p.window - tok0 : -1;
#pragma unroll
                    for (int q = 0; q < 32; ++q) {
                        if (token_at(q) > hi || token_at(q) <= lo) va[q] = 0xFF800000u;
                        if (token_at(q + 32) > hi || token_at(q + 32) <= lo) vb[q] = 0xFF800000u;
                    }
                }
                float mx = -INFINITY;
#pragma unroll
                for (int q = 0; q < 32; ++q) mx = fmax3(mx, __uint_as_float(va[q]), __uint_as_float(vb[q]));
                const float m_new = mx * sp;
                const bool need = m_new > m_used;
                if (moved || __any_sync(0xFFFFFFFFu, need)) {
                    if (!first) {
                        wait_pv(cX - 1u);
                        tc_fence_after();
                    }
                    const float alpha = need ? ex2(m_used - m_new) : 1.f;
                    if (need) m_used = m_new;
                    l *= alpha;
                    const float beta = BITS == 8 ? alpha * p8_pow2(ref_used - ref) : alpha;
                    ref_used = ref;
                    if (!first) {
#pragma unroll 1
                        for (int q = 0; q < D / 16; ++q) {
                            uint32_t o[16];
                            tmem_ld16(tO + 16u * q, o);
                            tc_wait_ld();
#pragma unroll
                            for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * beta);
                            tmem_st16(tO + 16u * q, o);
                        }
                    }
                }
                const unsigned long long sc2 = f2_pack(sp, sp), nm2 = f2_pack(BITS == 8 ? P_BIAS - m_used : -m_used, BITS == 8 ? P_BIAS - m_used : -m_used);
                unsigned long long ls2 = f2_pack(0.f, 0.f);
                softmax32(va, sc2, nm2, ls2, pk);
                tmem_st16(tSb, pk);
                softmax32(vb, sc2, nm2, ls2, pk);
                tmem_st16(tSb + 16u, pk);
                float l0, l1;
                f2_unpack(ls2, l0, l1);
                ls = l0 + l1;
            }
            l += ls;
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(C::PREADY + X * C::NBUF + (int)buf));
            ++cX;
            first = false;
        }
        it += (uint32_t)n;
        // ---- epilogue, the next unit's queries on their way meanwhile
        const bool full = u.kv0 == 0 && u.kv1 == u.en.pages, there = u.en.row0 + X * BM + row < u.en.n_rows;
        int i, h;
        page_row(p, min(u.en.row0 + X * BM + row, u.en.n_rows - 1), i, h);
        T* dst = (T*)p.out + ((size_t)(u.en.t0 + i) * p.q_heads + u.h * p.group + h) * D;
        float* part = w.part + ((size_t)blockIdx.x * 2 + (u.kv0 > 0 ? 0 : 1)) * C::PART;
        float4* pr = reinterpret_cast<float4*>(part) + X * BM + row;        // [D / 4 channels][256 rows]
        next_unit(w, u);
        if (u.valid && u.en.row0 + X * BM < u.en.n_rows) {
            fetch_queries<T, D>(p, u.en.t0, u.en.row0, u.en.n_rows, u.h, X, smem_u32(sQ));
            fetched = true;
        }
        wait_pv(cX - 1u);
        tc_fence_after();
        if (*c.abort_flag) l = __int_as_float(0x7FC00000);
        const float unit = BITS == 8 ? p8_pow2(ref_used) : 1.f, inv = l == 0.f ? 0.f : unit / l;
#pragma unroll 2
        for (int q = 0; q < D / 16; ++q) {
            uint32_t o[16];
            tmem_ld16(tO + 16u * q, o);
            tc_wait_ld();
            if (full) {
                if (there) {
                    uint32_t y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = page_result2<T>(__uint_as_float(o[2 * k]) * inv, __uint_as_float(o[2 * k + 1]) * inv);
                    reinterpret_cast<uint4*>(dst + 16 * q)[0] = make_uint4(y[0], y[1], y[2], y[3]);
                    reinterpret_cast<uint4*>(dst + 16 * q)[1] = make_uint4(y[4], y[5], y[6], y[7]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    pr[(4 * q + k) * 256] = make_float4(__uint_as_float(o[4 * k]) * unit, __uint_as_float(o[4 * k + 1]) * unit, __uint_as_float(o[4 * k + 2]) * unit,
                                                        __uint_as_float(o[4 * k + 3]) * unit);
            }
        }
        if (!full) reinterpret_cast<float2*>(part + 256 * D)[X * BM + row] = make_float2(m_used, l);
        tc_fence_before();
    }
}

// ------------------------------------------------------------------ MMA issue
// Tile x: S_k = Q K_k^T into buffer k % NBUF, then, once the softmax warps have turned it into P_k in place, O += P_k V_k.
// The pipe executes one thread's MMAs in order, so the QK of step k + NBUF goes out right behind the PV of step k into
// the buffer that this PV reads.
// Inlined: called, it cost 9 % of a frame's time (1374 tokens on 21 984: 235 us against 215).
template <int D>
__device__ __forceinline__ void mma_loop(const Work& w, const Cta c, Units u, const int x) {
    using C = Cfg<D>;
    auto BAR = [&](int i) { return c.bars + 8u * (uint32_t)i; };
    const uint32_t tS = c.tmem + C::tm_s(0, 0) + (uint32_t)x * (C::NBUF * 64), tO = c.tmem + C::tm_o(0) + (uint32_t)(x * D);
    const uint64_t qd = smem_desc(c.base + (uint32_t)x * C::Q_TILE);
    auto issue_qk = [&](uint32_t step, uint32_t buf) {
        const uint32_t st = step % C::NSTAGE;
        mbar_wait(BAR(C::KFULL + (int)st), (step / C::NSTAGE) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_K);
        tc_fence_after();
        const uint64_t kd = smem_desc(c.base + C::OFF_KV + st * C::STAGE);
        if (elect_one()) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                mma_ss(tS + buf * 64u, qd + (uint32_t)((k >> 2) * (16384 >> 4) + 2 * (k & 3)), kd + (uint32_t)((k >> 2) * (8192 >> 4) + 2 * (k & 3)), C::IDESC_QK, k > 0);
            tc_commit(BAR(C::SFULL + x * C::NBUF + (int)buf));
        }
        __syncwarp();
    };
    uint32_t it = 0, cT = 0, uT = 0;     // steps of the CTA; steps and units of this query tile
    for (; u.valid; next_unit(w, u)) {
        const int n = u.kv1 - u.kv0, ntile = u.en.row0 + BM < u.en.n_rows ? 2 : 1;
        if (x >= ntile) {
            // No second tile: this warp passes the stages' phases one by one and releases its share of each.  The stage is
            // not filled again before it has, so a parity wait here is never more than one phase late.
            for (int k = 0; k < n; ++k) {
                const uint32_t step = it + (uint32_t)k, st = step % C::NSTAGE;
                mbar_wait(BAR(C::KFULL + (int)st), (step / C::NSTAGE) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_K);
                mbar_wait(BAR(C::VFULL + (int)st), (step / C::NSTAGE) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_K);
                if (elect_one()) mbar_arrive(BAR(C::EMPTY + (int)st));      // (once every lane has passed)
            }
            it += (uint32_t)n;
            continue;
        }
        mbar_wait(BAR(C::QFULL + x), uT & 1u, c.abort_flag, c.status, XSV_DEV_SITE_Q);
        tc_fence_after();
        int qk = 0;
        for (; qk < C::NBUF && qk < n; ++qk) issue_qk(it + (uint32_t)qk, (cT + (uint32_t)qk) % C::NBUF);
        for (int k = 0; k < n; ++k) {
            const uint32_t step = it + (uint32_t)k, st = step % C::NSTAGE, cp = cT + (uint32_t)k, buf = cp % C::NBUF;
            mbar_wait(BAR(C::VFULL + (int)st), (step / C::NSTAGE) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_K);
            mbar_wait(BAR(C::PREADY + x * C::NBUF + (int)buf), (cp / C::NBUF) & 1u, c.abort_flag, c.status, XSV_DEV_SITE_P);
            tc_fence_after();
            const uint64_t vd = smem_desc(c.base + C::OFF_KV + st * C::STAGE + C::K_TILE);
            const uint32_t acc = k > 0 ? 1u : 0u;
            if (elect_one()) {
#pragma unroll
                for (int q = 0; q < 4; ++q)                // 16 tokens: 8 columns of P, 32 bytes of the value rows
                    mma_ts(tO, tS + buf * 64u + 8u * q, vd + 2u * q, C::IDESC_PV, q > 0 ? 1u : acc);
                tc_commit(BAR(C::PVDONE + x * C::NBUF + (int)buf));
                tc_commit(BAR(C::EMPTY + (int)st));
            }
            __syncwarp();
            if (qk < n) {
                issue_qk(it + (uint32_t)qk, (cT + (uint32_t)qk) % C::NBUF);
                ++qk;
            }
        }
        it += (uint32_t)n;
        cT += (uint32_t)n;
        ++uT;
    }
    // nothing of this warp's is in flight when the block ends, also where a wait ran out and no one else waits for it
    if (elect_one()) tc_commit(BAR(C::DRAIN + x));
    mbar_wait_bounded(BAR(C::DRAIN + x), 0u);
}

// ------------------------------------------------------------------ the kernel
__device__ __forceinline__ int owner(long long tick, long long total, int G) {     // CTA whose span holds the tick
    int b = (int)min((long long)(G - 1), tick * G / total);
    while (b + 1 < G && total * (b + 1) / G <= tick) ++b;
    while (b > 0 && total * b / G > tick) --b;
    return b;
}

template <typename T, int D, int BITS>
__global__ void __launch_bounds__(NTHREADS, 1) page_attn_tc5_kernel(const __grid_constant__ PageAttn p, const __grid_constant__ Work w) {
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t base = smem_u32(smem), bars = base + C::OFF_BAR;
    int* misc = reinterpret_cast<int*>(smem + C::OFF_BAR + C::COUNT * 8);          // tensor memory, abort, status, first entry, pages
    auto BAR = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, b = blockIdx.x;
    if (tid == 0) {
        for (int i = 0; i < C::NSTAGE; ++i) {
            mbar_init(BAR(C::KFULL + i), C::BLK);      // one arrival per slab
            mbar_init(BAR(C::VFULL + i), C::BLK);
            mbar_init(BAR(C::EMPTY + i), 2);           // one per query tile: a commit, or an arrival where there is no second tile
        }
        for (int i = 0; i < 2 * C::NBUF; ++i) {
            mbar_init(BAR(C::SFULL + i), 1);
            mbar_init(BAR(C::PREADY + i), 4);          // one arrival per softmax warp
            mbar_init(BAR(C::PVDONE + i), 1);
        }
        mbar_init(BAR(C::QFULL), 4);
        mbar_init(BAR(C::QFULL + 1), 4);
        mbar_init(BAR(C::DRAIN), 1);
        mbar_init(BAR(C::DRAIN + 1), 1);
        misc[1] = misc[2] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    xsv_dep_sync();
    const int entries = w.head[0];
    const long long total = *reinterpret_cast<const long long*>(w.head + 2);
    const int G = (int)max(1LL, min((long long)w.G, total / MIN_SPAN));            // CTAs that get a span
    if (b >= G || entries == 0) {                      // the same for the whole block
        if (tid == 0) w.desc[b] = make_int4(0, 0, 0, 0);
        return;
    }
    Units u;
    u.heads = p.pool.heads; u.entries = entries;
    u.t0 = total * b / G; u.t1 = total * (b + 1) / G;
    if (warp == 0) {                                   // the last entry that starts at or before the span
        int lo = 0, hi = entries;
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, i = lo + lane * step;
            const uint32_t in = __ballot_sync(0xFFFFFFFFu, i < hi && w.pre[i] * u.heads <= u.t0);
            lo += (31 - __clz((int)in)) * step;
            hi = min(hi, lo + step);
        }
        if (lane == 0) misc[3] = lo;
    }
    if (warp == 8 + NPROD + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t*)misc;
    u.e = misc[3];
    u.en = load_entry(w, u.e);
    {
        const long long in = u.t0 - w.pre[u.e] * u.heads;
        u.h = (int)min((long long)(u.heads - 1), in / u.en.ticks);
        u.base = w.pre[u.e] * u.heads + (long long)u.h * u.en.ticks;
    }
    settle(w, u);
    if (tid == 0) {
        // the first CTA that continues a unit describes how many parts it has
        int4 d = make_int4(0, 0, 0, 0);
        if (u.valid && u.kv0 > 0) {
            const long long step0 = u.base + COST_UNIT, step1 = step0 + (long long)(u.en.pages - 1) * step_cost(u.en);
            const int from = owner(step0, total, G), to = owner(step1, total, G);
            if (from == b - 1) d = make_int4(u.e, u.h, to - from + 1, 0);
        }
        w.desc[b] = d;
    }
    const Cta cta{smem, base, bars, tmem, misc + 1, misc + 2, smem_u32(misc + 4)};
    if (warp < 8) {
        softmax_loop<T, D, BITS>(p, w, cta, u);
    } else if (warp < 8 + NPROD) {
        if (BITS == 8) producer8_loop<T, D>(p, w, cta, u);
        else producer_loop<T, D>(p, w, cta, u);
    }
    else {
        mma_loop<D>(w, cta, u, warp - (8 + NPROD));
    }
    tc_fence_before();
    __syncthreads();
    xsv_dep_release();
    if (warp == 8 + NPROD + 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Units that several CTAs share, parts in the order of the CTAs.  Block: 16 rows x 16 groups of D / 16 channels.
template <typename T, int D>
__global__ void __launch_bounds__(256) page_attn_tc5_merge_kernel(const __grid_constant__ PageAttn p, const __grid_constant__ Work w) {
    using C = Cfg<D>;
    xsv_dep_release();
    xsv_dep_sync();
    const int b = blockIdx.x;
    const int4 d = w.desc[b];
    if (d.z == 0) return;
    const Entry en = load_entry(w, d.x);
    const int row = blockIdx.y * 16 + (threadIdx.x & 15), c = threadIdx.x >> 4, r = en.row0 + row;
    if (r >= en.n_rows) return;
    auto part = [&](int i) { return w.part + ((size_t)(b - 1 + i) * 2 + (i == 0 ? 1 : 0)) * C::PART; };
    float m = NO_MAX, l = 0.f;
    float4 o[D / 64];
#pragma unroll
    for (int k = 0; k < D / 64; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int i = 0; i < d.z; ++i) {
        const float* src = part(i);
        const float2 ml = reinterpret_cast<const float2*>(src + 256 * D)[row];
        const float mn = fmaxf(m, ml.x), a = ex2(m - mn), e = ex2(ml.x - mn);
        m = mn;
        l = l * a + ml.y * e;
#pragma unroll
        for (int k = 0; k < D / 64; ++k) {
            const float4 x = reinterpret_cast<const float4*>(src)[(16 * k + c) * 256 + row];
            o[k] = make_float4(o[k].x * a + x.x * e, o[k].y * a + x.y * e, o[k].z * a + x.z * e, o[k].w * a + x.w * e);
        }
    }
    int i, h;
    page_row(p, r, i, h);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* dst = (T*)p.out + ((size_t)(en.t0 + i) * p.q_heads + d.y * p.group + h) * D;
#pragma unroll
    for (int k = 0; k < D / 64; ++k)
        *reinterpret_cast<uint2*>(dst + 64 * k + 4 * c) = make_uint2(page_result2<T>(o[k].x * inv, o[k].y * inv), page_result2<T>(o[k].z * inv, o[k].w * inv));
}

// ------------------------------------------------------------------ host side
size_t max_entries(int n_tokens, int n_seqs, int group) { return (size_t)((long long)n_tokens * group / 256) + n_seqs + 1; }

template <typename T, int D, int BITS> cudaError_t launch(const PageAttn& p, const Work& w, cudaStream_t st) {
    static XsvPerDeviceInt ready;
    const int dev = xsv_current_device();
    if (!ready.get(dev)) {
        cudaError_t e = cudaFuncSetAttribute(page_attn_tc5_kernel<T, D, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<D>::SMEM);
        if (e != cudaSuccess) return e;
        ready.set(dev, 1);
    }
    cudaError_t e = xsv_launch_dep(page_list_kernel, dim3(1), dim3(1024), 0, st, p, w);
    if (e != cudaSuccess) return e;
    xsv_count_launch(1);
    e = xsv_launch_dep(page_attn_tc5_kernel<T, D, BITS>, dim3(w.G), dim3(NTHREADS), Cfg<D>::SMEM, st, p, w);
    if (e != cudaSuccess) return e;
    xsv_count_launch(1);
    e = xsv_launch_dep(page_attn_tc5_merge_kernel<T, D>, dim3(w.G, 16), dim3(256), 0, st, p, w);
    if (e == cudaSuccess) xsv_count_launch(1);
    return e;
}

}  // namespace

size_t xsv_page_tc5_workspace(int n_tokens, int n_seqs, int group, int head_dim) {
    const size_t G = (size_t)xsv_sm_count(), E = max_entries(n_tokens, n_seqs, group);
    return 256 + align256(G * sizeof(int4)) + align256((E + 1) * sizeof(long long)) + align256(E * sizeof(Entry)) + G * 2 * 256 * (head_dim + 2) * sizeof(float);
}

namespace {
template <int BITS> cudaError_t launch_any(const PageAttn& p, xsv_dtype dtype, int head_dim, void* workspace, cudaStream_t st) {
    Work w{};
    w.G = xsv_sm_count();
    const size_t E = max_entries(p.n_tokens, p.n_seqs, p.group);
    w.room = (int)E;
    char* at = (char*)workspace;
    w.head = (int*)at; at += 256;
    w.desc = (int4*)at; at += align256(w.G * sizeof(int4));
    w.pre = (long long*)at; at += align256((E + 1) * sizeof(long long));
    w.entry = (Entry*)at; at += align256(E * sizeof(Entry));
    w.part = (float*)at;
    if (dtype == XSV_F16) return head_dim == 64 ? launch<__half, 64, BITS>(p, w, st) : launch<__half, 128, BITS>(p, w, st);
    return head_dim == 64 ? launch<__nv_bfloat16, 64, BITS>(p, w, st) : launch<__nv_bfloat16, 128, BITS>(p, w, st);
}
}  // namespace

cudaError_t xsv_launch_page_tc5(const PageAttn& p, xsv_dtype dtype, int head_dim, void* workspace, cudaStream_t st) {
    return launch_any<4>(p, dtype, head_dim, workspace, st);
}
cudaError_t xsv_launch_page8_tc5(const PageAttn& p, xsv_dtype dtype, int head_dim, void* workspace, cudaStream_t st) {
    return launch_any<8>(p, dtype, head_dim, workspace, st);
}
