// Attention of few query rows a head over the 8-bit pages: out = softmax(scale s_k q C_k^T, causal, window) s_v C_v, with codes C
// and one scale a page for keys and values each; and attention of every new token over the pages that were selected for it.
//
// Bound by HBM, 2 d bytes a token and head, as long as a page's instructions take less than its bytes need to arrive:
//   - the products are taken transposed, S^T = C_k q^T and O^T = C_v^T P^T, so that the codes are the 16-row operand of
//     mma.m16n8k16 and a tile of 8 query rows (a group of query heads, or a few tokens of it) wastes none of it;
//   - every e4m3 value is an fp16 value: one conversion makes an operand register of two codes, values after one byte
//     permutation that brings two tokens of a channel together; the record's order makes that all there is (page8_layout.cuh);
//   - the scales are one factor a page: the keys' goes into the factor of the logits, the values' into the addition of the
//     page's sum to the output.
// q is scaled by a power of two per row so that its largest element lies in [1, 2).  The only roundings below float32 are those of
// q (fp16 inputs: none down to 2^-14 of a row's largest element; bf16: the same) and P to fp16 and of the result; a page is
// summed in the tensor cores and the pages by float32 additions, which round (the tensor cores' truncate).
//
// Work split.  Dense: a unit is (sequence, key/value head, tile of 8 NT query rows), its pages are the steps, and all steps are
// dealt in equal contiguous spans to the warps of the grid.  Selected: a unit is (token, head, tile of the group), with as many
// steps as the list has places.  A warp works alone (own page buffer in shared memory, filled by bulk copies, own softmax state): while
// it takes the products with a page's keys the values arrive, and the other way round.  A unit shared by several warps is
// merged by a second kernel in the order of the warps, so results do not depend on timing.
//
// Measured.  64 sequences of 900 to 16 000 tokens, one new token each, 32 query and 8 key/value heads of 128, bf16: 184 us, 6.0 TB/s (0.93 of the
// copy rate); 4 tokens over 200 001: 78 us, 5.2 TB/s; one sequence of 261, 16 heads of 64: 7.8 us with the merge, launch and latency.  Selected:
// 32 sequences, 32 pages a head: 33.9 us, 4.0 TB/s (4.6 pages a warp behind four loads that wait for one another); 509 tokens of
// one sequence, 24 pages each: 151 us, 10.6 TB/s out of L2, which bounds it (142 without the conversions, a third of 760 instructions a page).
#include <algorithm>
#include <cmath>

#include "../../include/xsv.h"
#include "page8_layout.cuh"
#include "page_attn.cuh"
#include "xsv_kernels.h"

namespace {

// Probabilities are 2^(x - m + P_BIAS), m a logit that was the row's maximum when it was last looked for: as long as none
// exceeds m by more than P_SLACK, m stays.  At most 2^10, they keep fp16's full significand down to 2^-20 of the maximum.
constexpr float P_BIAS = 6.f, P_SLACK = 4.f, NO_MAX = -1e30f;

struct Attn8 : PageAttn {
    int4* desc;          // [workers] units that begin to be shared: {first token, head, tile, parts << 8 | rows to write}; 0 parts: none
    float* part;         // [2 workers][slot] unnormalised rows
    // selected only
    const int* selected; // [n_tokens][heads][top]
    const int* seq;      // [n_tokens]
    const int* pos;      // [n_tokens]
    int top;
};

// one unnormalised tile: [NT][D / 16][32 lanes] float4, then maxima and sums [8 NT] float2
template <int D, int NT> struct Part { static constexpr int FLOATS = NT * (D / 16) * 128 + NT * 16; };

constexpr int WARPS = 4, THREADS = WARPS * 32;
template <int D, int NT> struct Shape {
    static constexpr int BLOCKS = D == 64 ? (NT == 1 ? 4 : 3) : (NT == 1 ? 3 : 2);
    static constexpr bool Q_REGS = NT == 1;
    static constexpr int PAGE_BYTES = Page8Rec<D>::K_BYTES + Page8Rec<D>::V_BYTES;
    static constexpr int PER_WARP = PAGE_BYTES + (Q_REGS ? 0 : NT * D * 16);
    static constexpr size_t SMEM = (size_t)WARPS * PER_WARP;
};

// A sequence as the split sees it (selected: a token).
struct Unit8 { int new_, total, p0, pages, tiles; };
template <bool SEL> __device__ __forceinline__ Unit8 unit_of(const Attn8& p, int s, int rows) {
    if constexpr (SEL) {
        Unit8 q{1, 0, 0, p.top, (p.group + rows - 1) / rows};
        const int seq = p.seq[s];
        if (seq >= 0 && seq < p.n_seqs) q.total = max(p.pos[s], -1) + 1;        // what the token sees
        return q;
    } else {
        const PageSeq x = page_seq(p, s);
        Unit8 q{x.new_, x.total, 0, 0, 0};
        q.p0 = p.window > 0 ? max(0, x.first - p.window + 1) / XSV_PAGE : 0;
        q.pages = max(1, (x.total + XSV_PAGE - 1) / XSV_PAGE - q.p0);
        const int n_rows = x.new_ * p.group;
        q.tiles = n_rows > p.row_limit ? 0 : (n_rows + rows - 1) / rows;
        return q;
    }
}

// A place in the list of steps: page `pg` of the `q.pages` of (sequence or token, head, tile).
struct Cursor { int s, head, tile, pg; Unit8 q; };
template <bool SEL> __device__ __forceinline__ void advance(const Attn8& p, Cursor& c, int rows) {
    if (++c.pg < c.q.pages) return;
    c.pg = 0;
    if (++c.tile < c.q.tiles) return;
    c.tile = 0;
    if (++c.head < p.pool.heads) return;
    c.head = 0;
    if constexpr (SEL) {
        if (++c.s < p.n_tokens) c.q = unit_of<SEL>(p, c.s, rows);
    } else {
        while (++c.s < p.n_seqs) {
            c.q = unit_of<SEL>(p, c.s, rows);
            if (c.q.tiles > 0) return;
        }
    }
}
// Token of the unit's first row; its query rows a head.
template <bool SEL> __device__ __forceinline__ int first_token(const Attn8& p, int s) { return SEL ? s : min(max(p.cu[s], 0), p.n_tokens); }

template <typename T, int D, int NT, bool SEL>
__global__ void __launch_bounds__(THREADS, Shape<D, NT>::BLOCKS) page8_attn_kernel(const __grid_constant__ Attn8 p) {
    using R = Page8Rec<D>;
    using S = Shape<D, NT>;
    constexpr int ROWS = 8 * NT, CT = D / 16, KB = D / 64;        // KB: 64-channel blocks
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) unsigned long long bars[WARPS][2];    // keys, values have arrived
    __shared__ long long s_base[THREADS + 1], s_warp[WARPS];
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    if (lane < 2) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&bars[wid][lane])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    xsv_dep_release();
    xsv_dep_sync();

    const int worker = blockIdx.x * WARPS + wid;
    long long steps;
    const int per = (p.n_seqs + THREADS - 1) / THREADS;
    if (SEL) {
        steps = (long long)p.n_tokens * p.pool.heads * ((p.group + ROWS - 1) / ROWS) * p.top;
        __syncwarp();
    } else {
        // steps of all sequences, scanned: thread i holds `per` consecutive sequences
        long long sum = 0;
        for (int s = tid * per; s < min(p.n_seqs, (tid + 1) * per); ++s) {
            const Unit8 q = unit_of<SEL>(p, s, ROWS);
            sum += (long long)p.pool.heads * q.tiles * q.pages;
        }
        long long x = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) s_warp[wid] = x;
        __syncthreads();
        long long before = x - sum;
        for (int w = 0; w < wid; ++w) before += s_warp[w];
        s_base[tid] = before;
        if (tid == THREADS - 1) s_base[THREADS] = before + sum;
        __syncthreads();
        steps = s_base[THREADS];
    }
    const int workers = (int)min((long long)gridDim.x * WARPS, steps);
    if (lane == 0) p.desc[worker] = make_int4(0, 0, 0, 0);
    if (worker >= workers) return;
    const long long x0 = steps * worker / workers, x1 = steps * (worker + 1) / workers;

    Cursor cur;
    {
        long long at;
        if (SEL) {
            const long long each = (long long)p.pool.heads * ((p.group + ROWS - 1) / ROWS) * p.top;
            cur.s = (int)(x0 / each);
            at = x0 - cur.s * each;
            cur.q = unit_of<SEL>(p, cur.s, ROWS);
        } else {
            int lo = 0, hi = THREADS - 1;                      // the last thread whose first step is at or before x0
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s_base[mid] <= x0) lo = mid; else hi = mid - 1;
            }
            at = x0 - s_base[lo];
            cur.s = lo * per;
            for (;; ++cur.s) {
                cur.q = unit_of<SEL>(p, cur.s, ROWS);
                const long long n = (long long)p.pool.heads * cur.q.tiles * cur.q.pages;
                if (at < n) break;
                at -= n;
            }
        }
        const int u = (int)(at / cur.q.pages);
        cur.pg = (int)(at - (long long)u * cur.q.pages);
        cur.head = u / cur.q.tiles;
        cur.tile = u - cur.head * cur.q.tiles;
        // The first worker that continues a unit describes how many parts it has.
        if (cur.pg > 0) {
            const long long unit0 = x0 - cur.pg, unit1 = unit0 + cur.q.pages;
            if (steps * (worker - 1) / workers <= unit0) {
                int last = worker;                             // the worker of the unit's last step
                long long k = (unit1 - 1) * workers / steps;
                if (k > last) last = (int)k;
                while (last + 1 < workers && steps * (last + 1) / workers < unit1) ++last;
                while (last > worker && steps * last / workers >= unit1) --last;
                const bool write = !SEL || cur.q.total > 0 || (p.seq[cur.s] >= 0 && p.seq[cur.s] < p.n_seqs);
                const int rows = write ? min(ROWS, cur.q.new_ * p.group - cur.tile * ROWS) : 0;
                if (lane == 0) p.desc[worker] = make_int4(first_token<SEL>(p, cur.s), cur.head, cur.tile, (last - worker + 2) << 8 | rows);
            }
        }
    }

    uint8_t* const keys = smem + wid * S::PER_WARP;
    uint8_t* const vals = keys + R::K_BYTES;
    const uint32_t k_bar = smem_u32(&bars[wid][0]), v_bar = smem_u32(&bars[wid][1]);
    // query operands: [n][64-channel block][2] of steps 2 i, 2 i + 1: {register 0, 1 of one, of the other}, this lane's
    uint4 q_regs[S::Q_REGS ? NT * KB * 2 : 1] = {};
    uint4* const q_smem = reinterpret_cast<uint4*>(vals + R::V_BYTES) + lane;
    auto query = [&](int i) { return S::Q_REGS ? q_regs[S::Q_REGS ? i : 0] : q_smem[i * 32]; };

    // The steps' pages, looked up 32 at a time, one a lane, a step ahead of the products: {page of the pool or -1, page of the
    // sequence}.
    Cursor ld = cur;
    int ld_left = (int)(x1 - x0), ids = -1, nos = 0, ids_from = -1;
    auto look_up = [&]() {
        ids_from = ld.pg & ~31;
        const int i = ids_from + lane;
        ids = -1;
        if (SEL) {
            if (i < p.top && ld.q.total > 0) {
                const int* list = p.selected + ((size_t)ld.s * p.pool.heads + ld.head) * p.top;
                nos = list[i];
                const int before = i > 0 ? list[i - 1] : -1;
                if (nos > before && nos >= 0 && nos < p.width && nos <= (ld.q.total - 1) / XSV_PAGE) ids = p.table[(size_t)p.seq[ld.s] * p.width + nos];
            }
        } else {
            nos = ld.q.p0 + i;
            if (i < ld.q.pages && nos < p.width && nos * XSV_PAGE < ld.q.total) ids = p.table[(size_t)ld.s * p.width + nos];
        }
        if ((unsigned long long)(long long)ids >= (unsigned long long)p.pool.n_pages) ids = -1;
    };
    int nx_page = -1, nx_no = 0;                               // the step at `ld`
    auto next = [&]() {
        if (ld_left == 0) return;
        if (ids_from < 0 || ld.pg < ids_from || ld.pg >= ids_from + 32) look_up();
        nx_page = __shfl_sync(0xFFFFFFFFu, ids, ld.pg & 31);
        nx_no = __shfl_sync(0xFFFFFFFFu, nos, ld.pg & 31);
    };
    auto bulk = [&](uint8_t* dst, const uint8_t* src, uint32_t bytes, uint32_t bar) {
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(bar) : "memory");
    };
    auto issue_keys = [&](int head, int page) {
        if (lane == 0 && page >= 0) bulk(keys, page8_rec<D>(p.pool, page, head) + R::K_CODES, R::K_BYTES, k_bar);
    };
    auto issue_vals = [&](int head, int page) {
        if (lane == 0 && page >= 0) bulk(vals, page8_rec<D>(p.pool, page, head) + R::V_CODES, R::V_BYTES, v_bar);
    };
    // page and number of the current step, and the head and page of the next one
    next();
    int page = nx_page, no = nx_no;
    issue_keys(ld.head, page);
    issue_vals(ld.head, page);
    auto step_ahead = [&]() {
        nx_page = -1;
        if (--ld_left > 0) {
            const int s = ld.s, head = ld.head;
            advance<SEL>(p, ld, ROWS);
            if (ld.s != s || (SEL && ld.head != head)) ids_from = -1;
            next();
        }
    };
    step_ahead();

    int parity = 0;                                            // of the barriers: copies of both halves come in pairs
    bool failed = false;
    // The warp gives up as one: what follows needs all of its lanes.  Nothing is issued any more then, and what is in flight on
    // the other barrier, if anything (its parity there: `other`), gets its time.
    auto wait = [&](uint32_t bar, uint32_t other_bar, int other, bool flies) {
        if (__all_sync(0xFFFFFFFFu, mbar_try(bar, parity)) || __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity))) return;
        failed = true;
        if (flies) mbar_wait_bounded(other_bar, other);
        __syncwarp();
    };
    float fac[NT][2], m[NT][2], l[NT][2], o[NT][CT][4];
    int qpos[NT][2], pos_lo = 0, pos_hi = 0;
    bool whole = false;                                        // the span holds the unit's first step
    const int n_steps = (int)(x1 - x0);
    for (int at = 0; at < n_steps; ++at) {
        const int head = cur.head, tile = cur.tile;
        if (at == 0 || cur.pg == 0) {
            // ---- a unit begins: its query rows
            whole = cur.pg == 0;
            const int n_rows = cur.q.new_ * p.group, t0 = first_token<SEL>(p, cur.s);
            int first = cur.q.total - cur.q.new_;
            if (!SEL && cur.q.total == p.width * XSV_PAGE) first = page_seq(p, cur.s).first;      // the sequence may go on beyond its table row
            {
                int i, h;
                page_row(p, tile * ROWS, i, h);
                pos_lo = first + i;
                page_row(p, min(n_rows, tile * ROWS + ROWS) - 1, i, h);
                pos_hi = first + i;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint4 raw[2 * KB];                             // channels 64 c + 16 j to + 15
                const int r = tile * ROWS + 8 * n + g;
                float mx = 0.f;
#pragma unroll
                for (int k = 0; k < 2 * KB; ++k) raw[k] = make_uint4(0, 0, 0, 0);
                if (r < n_rows) {
                    int i, h;
                    page_row(p, r, i, h);
                    const T* row = (const T*)p.Q + (size_t)(t0 + i) * p.q_stride + (size_t)(head * p.group + h) * D + 16 * j;
#pragma unroll
                    for (int k = 0; k < 2 * KB; ++k) raw[k] = *reinterpret_cast<const uint4*>(row + 64 * (k >> 1) + 8 * (k & 1));
                }
#pragma unroll
                for (int k = 0; k < 2 * KB; ++k)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 f = xsv_unpack2<T>(word(raw[k], w));
                        mx = fmaxf(mx, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
                // exponent that brings the largest element into [1, 2); two factors, since 2^-e alone may leave float32
                const int e = mx > 0.f ? max((__float_as_int(mx) >> 23) - 127, -126) : 0;
                const float s1 = pow2i(-(e / 2)), s2 = pow2i(-(e - e / 2));
#pragma unroll
                for (int k = 0; k < 2 * KB; ++k) {
                    uint32_t y[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 f = xsv_unpack2<T>(word(raw[k], w));
                        y[w] = pack_h2(f.x * s1 * s2, f.y * s1 * s2);
                    }
                    const uint4 x = make_uint4(y[0], y[1], y[2], y[3]);
                    if (S::Q_REGS) q_regs[S::Q_REGS ? n * 2 * KB + k : 0] = x;
                    else q_smem[(n * 2 * KB + k) * 32] = x;
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int er = __shfl_sync(0xFFFFFFFFu, e, 4 * (2 * j + c));
                    fac[n][c] = fmaxf(p.scale * pow2i(er), MIN_FACTOR);
                    const int row = tile * ROWS + 8 * n + 2 * j + c;
                    int i, h;
                    page_row(p, row, i, h);
                    qpos[n][c] = row < n_rows ? first + i : -1;
                    m[n][c] = NO_MAX;
                    l[n][c] = 0.f;
                }
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[n][c][i] = 0.f;
            }
        }
        // ---- the step's page
        const int tok0 = no * XSV_PAGE;
        if (page >= 0 && !failed) wait(k_bar, v_bar, parity, true);
        if (page >= 0 && !failed) {
            const int seen = cur.q.total - tok0;               // tokens of the page that there are
            const bool part = seen < XSV_PAGE;
            const bool mask = tok0 + XSV_PAGE - 1 > pos_lo || part || (p.window > 0 && tok0 <= pos_hi - p.window);
            const float2 scales = *reinterpret_cast<const float2*>(keys + R::PARAMS);
            float s[NT][4][4], f[NT][2];
#pragma unroll
            for (int c = 0; c < KB; ++c) {
                uint4 q[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) { q[n][0] = query((n * KB + c) * 2); q[n][1] = query((n * KB + c) * 2 + 1); }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint4 ra = *reinterpret_cast<const uint4*>(keys + ((2 * t * KB + c) * 32 + lane) * 16);
                    const uint4 rb = *reinterpret_cast<const uint4*>(keys + (((2 * t + 1) * KB + c) * 32 + lane) * 16);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t a0, a1, a2, a3;
                        p8_halves(word(ra, w), a0, a2);
                        p8_halves(word(rb, w), a1, a3);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint32_t b0 = word(q[n][w >> 1], 2 * (w & 1)), b1 = word(q[n][w >> 1], 2 * (w & 1) + 1);
                            if (c == 0 && w == 0) mma0(s[n][t], a0, a1, a2, a3, b0, b1);
                            else mma(s[n][t], a0, a1, a2, a3, b0, b1);
                        }
                    }
                }
            }
            __syncwarp();
            issue_keys(ld.head, nx_page);                      // the next step's, into the same place
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) f[n][c] = fmaxf(fac[n][c] * scales.x, MIN_FACTOR);
            if (mask) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int tok = tok0 + 16 * t + g + 8 * (i >> 1), at_q = qpos[n][i & 1];
                            const bool in = tok <= at_q && (p.window <= 0 || tok > at_q - p.window) && tok < cur.q.total;
                            if (!in) s[n][t][i] = -INFINITY;   // whatever stood there, NaN included
                        }
            }
            // ---- maximum: looked for only when a logit exceeds the one in use
            float xm[NT][2];
            bool raise = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = fmaxf(s[n][0][c], s[n][0][c + 2]);
#pragma unroll
                    for (int t = 1; t < 4; ++t) x = fmax3(x, s[n][t][c], s[n][t][c + 2]);
                    xm[n][c] = x * f[n][c];
                    raise = raise || xm[n][c] > m[n][c] + P_SLACK;
                }
            if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float x = xm[n][c];
                        x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 16));
                        x = fmaxf(x, m[n][c]);
                        const float a = ex2(m[n][c] - x);
                        m[n][c] = x;
                        l[n][c] *= a;
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) { o[n][ct][c] *= a; o[n][ct][c + 2] *= a; }
                    }
            }
            // ---- probabilities, as the products' second operand: tokens 16 t + {2 j, 2 j + 1} (+ 8), row g; their sums
            uint32_t b[4][NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float off0 = P_BIAS - m[n][0], off1 = P_BIAS - m[n][1];
                float sum[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    b[t][n][0] = transpose8(pack_h2(ex2(fmaf(s[n][t][0], f[n][0], off0)), ex2(fmaf(s[n][t][1], f[n][1], off1))));
                    b[t][n][1] = transpose8(pack_h2(ex2(fmaf(s[n][t][2], f[n][0], off0)), ex2(fmaf(s[n][t][3], f[n][1], off1))));
                    constexpr uint32_t ONES = 0x3C003C00u;
                    if (t == 0) mma0(sum, ONES, ONES, ONES, ONES, b[0][n][0], b[0][n][1]);
                    else mma(sum, ONES, ONES, ONES, ONES, b[t][n][0], b[t][n][1]);
                }
                l[n][0] += sum[0];
                l[n][1] += sum[1];
            }
            // ---- its values, half of a lane's channels after the other where two tiles' sums would not fit the registers
            wait(v_bar, k_bar, parity ^ 1, nx_page >= 0);
            if (!failed) {
                constexpr int HALVES = D == 128 && NT == 2 ? 2 : 1, WV = D / 32 / HALVES;       // words of a piece at a time
#pragma unroll
                for (int half = 0; half < HALVES; ++half) {
                    float acc[NT][2 * WV][4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        uint32_t x[2][2][WV];                  // [b][h], tokens 16 t + 8 b + 2 j + h
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint8_t* at_v = vals + ((4 * t + i) * 32 + lane) * (D / 8) + 4 * WV * half;
                            if (WV == 4) {
                                const uint4 y = *reinterpret_cast<const uint4*>(at_v);
#pragma unroll
                                for (int w = 0; w < WV; ++w) x[i >> 1][i & 1][w] = word(y, w);
                            } else {
                                const uint2 y = *reinterpret_cast<const uint2*>(at_v);
                                x[i >> 1][i & 1][0] = y.x;
                                x[i >> 1][i & 1][1] = y.y;
                            }
                        }
                        if (part) {                            // places that hold no token: no bits of theirs count
                            asm volatile("" ::: "memory");     // a branch: as predicated code it would cost every page
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (16 * t + 8 * (i >> 1) + 2 * j + (i & 1) >= seen)
#pragma unroll
                                    for (int w = 0; w < WV; ++w) x[i >> 1][i & 1][w] = 0u;
                        }
#pragma unroll
                        for (int w = 0; w < WV; ++w) {
                            uint32_t e[2][4];                  // channels 4 w to 4 w + 3 of both b
#pragma unroll
                            for (int bb = 0; bb < 2; ++bb) {
                                p8_halves(__byte_perm(x[bb][0][w], x[bb][1][w], 0x5140), e[bb][0], e[bb][1]);
                                p8_halves(__byte_perm(x[bb][0][w], x[bb][1][w], 0x7362), e[bb][2], e[bb][3]);
                            }
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                if (t == 0) {
                                    mma0(acc[n][2 * w], e[0][0], e[0][1], e[1][0], e[1][1], b[0][n][0], b[0][n][1]);
                                    mma0(acc[n][2 * w + 1], e[0][2], e[0][3], e[1][2], e[1][3], b[0][n][0], b[0][n][1]);
                                } else {
                                    mma(acc[n][2 * w], e[0][0], e[0][1], e[1][0], e[1][1], b[t][n][0], b[t][n][1]);
                                    mma(acc[n][2 * w + 1], e[0][2], e[0][3], e[1][2], e[1][3], b[t][n][0], b[t][n][1]);
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 2 * WV; ++i)
#pragma unroll
                            for (int c = 0; c < 4; ++c) o[n][2 * WV * half + i][c] = fmaf(acc[n][i][c], scales.y, o[n][2 * WV * half + i][c]);
                }
                __syncwarp();
                issue_vals(ld.head, nx_page);
            }
            parity ^= 1;
        } else if (!failed) {                                  // no page here: nothing of this step's is in flight
            issue_keys(ld.head, nx_page);
            issue_vals(ld.head, nx_page);
        }

        // ---- the unit, or this span's part of it, is done
        const bool ends = cur.pg + 1 == cur.q.pages;
        if (ends || at + 1 == n_steps) {
            if (failed)
#pragma unroll
                for (int n = 0; n < NT; ++n) l[n][0] = l[n][1] = NAN;
            if (whole && ends) {
                const int n_rows = cur.q.new_ * p.group, t0 = first_token<SEL>(p, cur.s);
                const bool write = !SEL || cur.q.total > 0 || (p.seq[cur.s] >= 0 && p.seq[cur.s] < p.n_seqs);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int r = tile * ROWS + 8 * n + 2 * j + c;
                        if (r >= n_rows || !write) continue;
                        int i, h;
                        page_row(p, r, i, h);
                        const float inv = l[n][c] == 0.f ? 0.f : 1.f / l[n][c];
                        T* dst = (T*)p.out + ((size_t)(t0 + i) * p.q_heads + head * p.group + h) * D + (D / 8) * g;
#pragma unroll
                        for (int v = 0; v < CT / 4; ++v)
                            *reinterpret_cast<uint4*>(dst + 8 * v) = make_uint4(
                                page_result2<T>(o[n][4 * v][c] * inv, o[n][4 * v][c + 2] * inv), page_result2<T>(o[n][4 * v + 1][c] * inv, o[n][4 * v + 1][c + 2] * inv),
                                page_result2<T>(o[n][4 * v + 2][c] * inv, o[n][4 * v + 2][c + 2] * inv), page_result2<T>(o[n][4 * v + 3][c] * inv, o[n][4 * v + 3][c + 2] * inv));
                    }
            } else {
                float* dst = p.part + (size_t)(2 * worker + (whole ? 1 : 0)) * Part<D, NT>::FLOATS;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
                        reinterpret_cast<float4*>(dst)[(n * CT + ct) * 32 + lane] = make_float4(o[n][ct][0], o[n][ct][1], o[n][ct][2], o[n][ct][3]);
                    if (g == 0)
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            reinterpret_cast<float2*>(dst + NT * CT * 128)[8 * n + 2 * j + c] = make_float2(m[n][c], l[n][c]);
                }
            }
        }
        if (at + 1 < n_steps) {
            advance<SEL>(p, cur, ROWS);
            page = nx_page;
            no = nx_no;
            step_ahead();
        }
    }
}

// Units that several warps share.  A block of 8 warps looks at the descriptions of 16 workers and merges 16 channels of the units that
// begin to be shared there: as many warps a unit as there are for it, which take its parts in turn and are merged in their order; a lane has
// 4 values (2 rows x 2 channels).  (The whole block for one unit after the other: 15 us instead of 5 where most units have two parts.)
// (One warp for all channels of a unit: 147 instead of 151 us where a unit has at most two parts, 211 instead of 184 and 45 instead of 34 where
// there are more.)  Measured with and without the second launch, it costs one
// sequence of 261 2.3 us, 64 sequences and 4 tokens over 200 001 7.5, 32 selecting sequences 5.4, 509 selecting tokens 8.7: its launch, its
// descriptions' and then its parts' latency.
constexpr int MERGE_UNITS = 16, MERGE_WARPS = 8;
template <typename T, int D, int NT>
__global__ void __launch_bounds__(MERGE_WARPS * 32) page8_attn_merge_kernel(const __grid_constant__ Attn8 p, int workers) {
    constexpr int ROWS = 8 * NT, CT = D / 16, PF = Part<D, NT>::FLOATS;
    __shared__ float4 s_o[MERGE_WARPS][32], s_ml[MERGE_WARPS][32];
    xsv_dep_release();
    xsv_dep_sync();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, n = blockIdx.y / CT, ct = blockIdx.y % CT;
    const int g = lane >> 2, j = lane & 3, r0 = 8 * n + 2 * j;
    struct Acc {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f), ml = make_float4(NO_MAX, 0.f, NO_MAX, 0.f);
        __device__ __forceinline__ void add(const float4& x, const float4& y) {      // y: maximum and sum of both rows
            const float m0 = fmaxf(ml.x, y.x), m1 = fmaxf(ml.z, y.z);
            const float a0 = ex2(ml.x - m0), b0 = ex2(y.x - m0), a1 = ex2(ml.z - m1), b1 = ex2(y.z - m1);
            o.x = o.x * a0 + x.x * b0; o.z = o.z * a0 + x.z * b0;
            o.y = o.y * a1 + x.y * b1; o.w = o.w * a1 + x.w * b1;
            ml = make_float4(m0, ml.y * a0 + y.y * b0, m1, ml.w * a1 + y.w * b1);
        }
    };
    const int w0 = blockIdx.x * MERGE_UNITS;
    int4 mine = make_int4(0, 0, 0, 0);
    if (lane < MERGE_UNITS && w0 + lane < workers) mine = p.desc[w0 + lane];
    auto unit = [&](int from) { return make_int4(__shfl_sync(0xFFFFFFFFu, mine.x, from), __shfl_sync(0xFFFFFFFFu, mine.y, from), __shfl_sync(0xFFFFFFFFu, mine.z, from), __shfl_sync(0xFFFFFFFFu, mine.w, from)); };
    auto sum = [&](Acc& acc, int w, int parts, int i0, int step) {
        constexpr int AHEAD = 4;                                // parts on their way together (8: 3 % slower where units have few)
        for (int i = i0; i < parts; i += AHEAD * step) {
            float4 x[AHEAD], y[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int at = i + k * step;
                x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                y[k] = make_float4(NO_MAX, 0.f, NO_MAX, 0.f);
                if (at < parts) {
                    const float* part = p.part + (size_t)(at == 0 ? 2 * (w - 1) + 1 : 2 * (w + at - 1)) * PF;
                    x[k] = reinterpret_cast<const float4*>(part)[(n * CT + ct) * 32 + lane];
                    y[k] = *reinterpret_cast<const float4*>(part + NT * CT * 128 + 2 * r0);
                }
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i + k * step < parts) acc.add(x[k], y[k]);
        }
    };
    auto write = [&](const Acc& acc, const int4& d) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (r0 + c >= (d.w & 255)) continue;
            const int r = d.z * ROWS + r0 + c;
            int i, h;
            page_row(p, r, i, h);
            const float l = c ? acc.ml.w : acc.ml.y, inv = l == 0.f ? 0.f : 1.f / l;
            T* dst = (T*)p.out + ((size_t)(d.x + i) * p.q_heads + d.y * p.group + h) * D + (D / 8) * g + 2 * ct;
            *reinterpret_cast<uint32_t*>(dst) = page_result2<T>((c ? acc.o.y : acc.o.x) * inv, (c ? acc.o.w : acc.o.z) * inv);
        }
    };
    const uint32_t todo = __ballot_sync(0xFFFFFFFFu, mine.w > 0);                // the same for the whole block
    const int units = __popc(todo), per = units <= 1 ? 8 : units == 2 ? 4 : units <= 4 ? 2 : 1;      // warps of a unit
    for (int at = wid / per; at < (per == 1 ? units : MERGE_WARPS / per); at += MERGE_WARPS / per) {
        Acc acc;
        int from = 0;
        int4 d = make_int4(0, 0, 0, 0);
        if (at < units) {
            uint32_t rest = todo;
            for (int i = 0; i < at; ++i) rest &= rest - 1;
            from = __ffs(rest) - 1;
            d = unit(from);
            sum(acc, w0 + from, d.w >> 8, wid % per, per);
        }
        if (per > 1) {                                          // once: every warp has one unit or none
            s_o[wid][lane] = acc.o;
            s_ml[wid][lane] = acc.ml;
            __syncthreads();
            if (at >= units || wid % per != 0) return;
            for (int i = 1; i < per; ++i) acc.add(s_o[wid + i][lane], s_ml[wid + i][lane]);
        }
        write(acc, d);
    }
}

// ------------------------------------------------------------------ host side
template <int D, int NT> int workers_at() { return xsv_sm_count() * Shape<D, NT>::BLOCKS * WARPS; }
int workers_of(int head_dim, int nt) {
    return head_dim == 64 ? (nt == 1 ? workers_at<64, 1>() : workers_at<64, 2>()) : (nt == 1 ? workers_at<128, 1>() : workers_at<128, 2>());
}
// 8 query rows a tile where a head has no more, else 16
int tiles_of(long long rows) { return rows <= 8 ? 1 : 2; }

// Sequences with more query rows a head go to the tensor-memory kernel, whose time does not depend on them up to 128.
// 8 sequences of 8000 tokens, this kernel against that one: 16 heads of 64, 64 rows 92 against 98 us, 80 rows 112 against 99; 8
// key/value heads of 128, 32 rows 60 against 74, 48 rows 70 against 75, 64 rows 87 against 75.
int few_rows(int head_dim) { return head_dim == 64 ? 64 : 48; }
bool many_rows(int max_new, int group, int head_dim) { return (long long)max_new * group > few_rows(head_dim); }
// ... unless there is so little to do that its launches and its units' begins and ends, 28 to 40 us, are most of it.  What bounds the work is
// known on the host: pages that the table has room for, times tiles of 16 rows.  This kernel against that one: heads of 128, a bound of 1584 19 us
// against 38, 8448 34 against 39, 9696 37 against 39, 16 448 54 against 40; heads of 64, 4608 20 against 33, 14 784 35 against 36, 20 736 40 against 36.
bool little_work(int n_tokens, int n_seqs, int group, int heads, int width, int head_dim) {
    return ((long long)n_tokens * group / 16 + n_seqs) * heads * width <= (head_dim == 64 ? 14336 : 8960);
}

size_t few_space(int nt, int head_dim) {
    const size_t workers = (size_t)workers_of(head_dim, nt), pf = (size_t)nt * (head_dim / 16) * 128 + nt * 16;
    return align256(workers * sizeof(int4)) + align256(2 * workers * pf * sizeof(float));
}
size_t workspace_of(int n_tokens, int n_seqs, int max_new, int group, int head_dim) {
    return few_space(tiles_of((long long)max_new * group), head_dim) + (many_rows(max_new, group, head_dim) ? xsv_page_tc5_workspace(n_tokens, n_seqs, group, head_dim) : 0);
}

template <typename T, int D, int NT, bool SEL> cudaError_t launch(Attn8& p, cudaStream_t st) {
    auto kernel = page8_attn_kernel<T, D, NT, SEL>;
    constexpr size_t smem = Shape<D, NT>::SMEM;
    static XsvPerDeviceInt ready;
    const int dev = xsv_current_device();
    if (!ready.get(dev)) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        ready.set(dev, 1);
    }
    const int grid = xsv_sm_count() * Shape<D, NT>::BLOCKS, workers = workers_at<D, NT>();
    cudaError_t e = xsv_launch_dep(kernel, dim3(grid), dim3(THREADS), smem, st, p);
    if (e != cudaSuccess) return e;
    xsv_count_launch(1);
    e = xsv_launch_dep(page8_attn_merge_kernel<T, D, NT>, dim3((workers + MERGE_UNITS - 1) / MERGE_UNITS, NT * (D / 16)), dim3(MERGE_WARPS * 32), 0, st, p, workers);
    if (e == cudaSuccess) xsv_count_launch(1);
    return e;
}
template <bool SEL> cudaError_t launch_any(Attn8& p, xsv_dtype dtype, int head_dim, int nt, cudaStream_t st) {
    auto with = [&](auto zero) {
        using T = decltype(zero);
        if (head_dim == 64) return nt == 1 ? launch<T, 64, 1, SEL>(p, st) : launch<T, 64, 2, SEL>(p, st);
        return nt == 1 ? launch<T, 128, 1, SEL>(p, st) : launch<T, 128, 2, SEL>(p, st);
    };
    return dtype == XSV_F16 ? with(__half{}) : with(__nv_bfloat16{});
}

void set_group(Attn8& p, int q_heads, int kv_heads) {
    p.q_heads = q_heads;
    p.group = q_heads / kv_heads;
    p.group_shift = -1;
    for (int b = 0; b < 16; ++b) if (p.group == 1 << b) p.group_shift = b;
}
bool heads_fit(int q_heads, int kv_heads) { return kv_heads > 0 && q_heads >= kv_heads && q_heads % kv_heads == 0 && q_heads <= 1 << 16; }

}  // namespace

extern "C" size_t xsv_page8_attention_workspace(int n_tokens, int n_seqs, int max_new, int q_heads, int kv_heads, int head_dim) {
    if (n_tokens <= 0 || n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS || max_new <= 0) return 0;
    if (!heads_fit(q_heads, kv_heads) || (head_dim != 64 && head_dim != 128)) return 0;
    return workspace_of(n_tokens, n_seqs, std::min(max_new, n_tokens), q_heads / kv_heads, head_dim);
}

extern "C" xsv_status xsv_page8_attention(const xsv_page8_pool* pool, const void* Q, long long q_stride, int n_tokens, int q_heads, const int* block_table,
                                          int table_width, const int* cu_new, const int* total_len, const int* slot_map, int n_seqs, int max_new,
                                          float scale, int window, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    Attn8 p{};
    xsv_status s = xsv_page8_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_tokens < 0 || n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS || table_width <= 0 || max_new < 0 || window < 0) return XSV_ERR_ARG;
    if (!heads_fit(q_heads, pool->kv_heads)) return XSV_ERR_ARG;
    if (!(scale > 0.f) || !std::isfinite(scale)) return XSV_ERR_ARG;
    if (n_tokens == 0 || max_new == 0) return XSV_OK;
    if (max_new > n_tokens) max_new = n_tokens;
    if (!Q || !block_table || !cu_new || !total_len || !out || !workspace) return XSV_ERR_ARG;
    if (n_tokens > 1 && q_stride < (long long)q_heads * pool->head_dim) return XSV_ERR_ARG;
    if (((uintptr_t)Q | (uintptr_t)out | (uintptr_t)workspace) & 15 || q_stride & 7) return XSV_ERR_SHAPE;
    set_group(p, q_heads, pool->kv_heads);
    // rows of a sequence and its tokens are 32-bit numbers
    if ((long long)n_tokens * p.group > 1LL << 30 || (long long)table_width * XSV_PAGE > 1LL << 30) return XSV_ERR_LIMIT;
    if (workspace_bytes < workspace_of(n_tokens, n_seqs, max_new, p.group, pool->head_dim)) return XSV_ERR_ARG;
    const int nt = tiles_of((long long)max_new * p.group);
    p.Q = Q; p.out = out; p.table = block_table; p.cu = cu_new; p.total = total_len; p.slot = slot_map; p.q_stride = q_stride;
    p.desc = (int4*)workspace;
    p.part = (float*)((char*)workspace + align256((size_t)workers_of(pool->head_dim, nt) * sizeof(int4)));
    p.scale = scale * 1.4426950408889634f;
    p.width = table_width; p.n_seqs = n_seqs; p.n_tokens = n_tokens;
    p.window = window;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    p.row_limit = 1 << 30;
    if (many_rows(max_new, p.group, pool->head_dim) && !little_work(n_tokens, n_seqs, p.group, pool->kv_heads, table_width, pool->head_dim)) {
        p.row_limit = n_seqs == 1 ? 0 : few_rows(pool->head_dim);
        e = xsv_launch_page8_tc5(p, pool->dtype, pool->head_dim, (char*)workspace + few_space(nt, pool->head_dim), st);
    }
    if (e == cudaSuccess && p.row_limit > 0) e = launch_any<false>(p, pool->dtype, pool->head_dim, nt, st);
    return e == cudaSuccess ? XSV_OK : xsv_cuda_status(e);
}

extern "C" size_t xsv_page8_attention_selected_workspace(int q_heads, int kv_heads, int head_dim) {
    if (!heads_fit(q_heads, kv_heads) || (head_dim != 64 && head_dim != 128)) return 0;
    return few_space(tiles_of(q_heads / kv_heads), head_dim);
}

extern "C" xsv_status xsv_page8_attention_selected(const xsv_page8_pool* pool, const void* Q, long long q_stride, int n_tokens, int q_heads,
                                                   const int* block_table, int table_width, int n_seqs, const int* token_seq, const int* positions,
                                                   const int* selected, int top, float scale, void* out, void* workspace, size_t workspace_bytes,
                                                   void* stream) {
    Attn8 p{};
    xsv_status s = xsv_page8_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_tokens < 0 || n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS || table_width <= 0 || top <= 0) return XSV_ERR_ARG;
    if (!heads_fit(q_heads, pool->kv_heads)) return XSV_ERR_ARG;
    if (!(scale > 0.f) || !std::isfinite(scale)) return XSV_ERR_ARG;
    if (n_tokens == 0) return XSV_OK;
    if (!Q || !block_table || !token_seq || !positions || !selected || !out || !workspace) return XSV_ERR_ARG;
    if (n_tokens > 1 && q_stride < (long long)q_heads * pool->head_dim) return XSV_ERR_ARG;
    if (((uintptr_t)Q | (uintptr_t)out | (uintptr_t)workspace) & 15 || q_stride & 7) return XSV_ERR_SHAPE;
    set_group(p, q_heads, pool->kv_heads);
    if ((long long)n_tokens * p.group > 1LL << 30 || (long long)table_width * XSV_PAGE > 1LL << 30 || top > XSV_PAGE8_MAX_TOP) return XSV_ERR_LIMIT;
    // a worker's span is a 32-bit number of steps
    const int nt = tiles_of(p.group);
    const long long units = (long long)n_tokens * pool->kv_heads * ((p.group + 8 * nt - 1) / (8 * nt));
    if (units > 1LL << 30) return XSV_ERR_LIMIT;
    if (workspace_bytes < few_space(nt, pool->head_dim)) return XSV_ERR_ARG;
    p.Q = Q; p.out = out; p.table = block_table; p.q_stride = q_stride;
    p.selected = selected; p.seq = token_seq; p.pos = positions; p.top = top;
    p.desc = (int4*)workspace;
    p.part = (float*)((char*)workspace + align256((size_t)workers_of(pool->head_dim, nt) * sizeof(int4)));
    p.scale = scale * 1.4426950408889634f;
    p.width = table_width; p.n_seqs = n_seqs; p.n_tokens = n_tokens;
    const cudaError_t e = launch_any<true>(p, pool->dtype, pool->head_dim, nt, (cudaStream_t)stream);
    return e == cudaSuccess ? XSV_OK : xsv_cuda_status(e);
}
