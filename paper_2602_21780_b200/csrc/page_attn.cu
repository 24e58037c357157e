// Attention of few query rows a head over the 4-bit pages: out = softmax(scale q K^T, causal, window) V with
// K = code s + z per channel, V = code s + z per token.
//
// Bound by HBM (1.125 d bytes a token and head) as long as the instructions a token costs stay below what its bytes
// take to arrive; everything here serves that:
//   - the products are taken transposed, S^T = K q^T and O^T = V^T P^T, so that the codes are the 16-row operand of
//     mma.m16n8k16 and a tile of 8 query rows (a group of query heads, or a few tokens of it) wastes none of it;
//   - codes go to the tensor cores as fp16 subnormals, one mask per two codes (page_layout.cuh); the parameters
//     are folded into the other operand: s of a channel into q (once a page, 16 rows x d products instead of 64 x d),
//     s of a token into P; z enters as one more product, q . z (added to all of S) and sum_t p_t z_t (added to all
//     channels of O);
//   - P^T comes out of S^T by one movmatrix per 8 x 8 block, O^T leaves with 8 consecutive channels a lane.
// q is scaled by a power of two per row so that its largest element lies in [2, 4): with s <= 8734, q s never leaves fp16,
// and elements below 2^-14 lose at most 2^-25 absolutely.  s is scaled by a power of two per page where that keeps P s inside
// fp16's range whatever the values' magnitude.  The roundings below float32 are those of q s, P and P s to fp16 (the tensor
// cores' operands; 2^-12 of a factor on average, for fp16 results taken around the codes' middle) and of the result; sums,
// maxima and the output accumulate in float32.
//
// Work split.  A unit is (sequence, key/value head, tile of 8 NT query rows); its pages are the steps.  All steps of all
// units are dealt in equal contiguous spans to the warps of the grid, so ragged lengths and few sequences fill the GPU
// alike; a warp works alone (own ring of page records in shared memory, filled by bulk copies, own softmax state), no
// block-wide barrier in the loop.  A unit shared by several warps is merged by a second kernel in the order of the
// warps, so results do not depend on timing.  Each block finds its spans itself by scanning the lengths.
//
// Measured.  64 sequences of 900 to 16 000 tokens, one new token each, 32 query and 8 key/value heads of 128, bf16: 127 us,
// 4.95 TB/s of 6.57 (first version 159).  Without its arithmetic this kernel takes some 110 us, without its loads 115.  No
// unit is saturated (DRAM 81 %, ALU 55 %, issue slots 54 %): with 11 warps a multiprocessor, 880 instructions a page each
// (333 unpack, 80 products, the rest parameters, softmax and bookkeeping), the latencies of both are not hidden.
// 4 tokens (16 rows) over one sequence of 200 001: 75 us, 3.1 TB/s; its 64 accumulators leave 2 warps a scheduler, and
// issue slots 41 %, tensor pipe 45 % busy.
// One sequence of 261 tokens, 16 heads of 64: 8.8 us with the merge, launch and latency.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/xsv.h"
#include "page_attn.cuh"
#include "tc5_ptx.cuh"
#include "xsv_kernels.h"

namespace {

// Probabilities are 2^(x - m + P_BIAS) with m a logit that was the row's maximum when it was last looked for: as long as
// none exceeds m by more than P_SLACK, m stays (one vote instead of a reduction and a rescale).  At most 2^10, they
// keep fp16's full significand down to 2^-20 of the row's maximum; times a value scale of at most 16 they stay in range.
constexpr float P_BIAS = 6.f, P_SLACK = 4.f, NO_MAX = -1e30f;

struct Attn : PageAttn {
    int4* desc;          // [workers] units that are shared: {sequence, head, tile, parts}; parts 0: none begins to be shared here
    float* part;         // [2 workers][slot] unnormalised rows
};

// one unnormalised tile: [NT][D / 16][32 lanes] float4, then maxima and sums [8 NT] float2
template <int D, int NT> struct Part { static constexpr int FLOATS = NT * (D / 16) * 128 + NT * 16; };

// Blocks per multiprocessor and stages (page records) per warp: as many warps as the registers allow (the tile's
// accumulators set them: 16 warps of 128, 12 of 168, 8 of 255), as many stages as shared memory then does.  A tile of 16 rows
// keeps its query operands in shared memory.  (16 warps of half-page stages and spilled registers at head_dim 128: 178 us
// instead of 142 for 64 sequences.)
constexpr int WARPS = 4, THREADS = WARPS * 32;
template <int D, int NT> struct Shape {
    static constexpr int BLOCKS = D == 64 ? (NT == 1 ? 4 : 3) : (NT == 1 ? 3 : 2);
    static constexpr int STAGES = D == 64 ? 3 : 2;
    static constexpr bool Q_REGS = NT == 1;
    static constexpr int PER_WARP = STAGES * PageRec<D>::BYTES + (Q_REGS ? 0 : NT * D * 16);
    static constexpr size_t SMEM = (size_t)WARPS * PER_WARP;
};

__device__ __forceinline__ uint32_t hfnma2_u(uint32_t a, uint32_t b, uint32_t c) {      // c - a b
    const __half2 r = __hfma2(__hneg2(*reinterpret_cast<__half2*>(&a)), *reinterpret_cast<__half2*>(&b), *reinterpret_cast<__half2*>(&c));
    return *reinterpret_cast<const uint32_t*>(&r);
}
constexpr uint32_t ONES = 0x3C003C00u, EIGHTS = 0x48004800u, MINUS_EIGHTS = 0xC800C800u;   // pairs of fp16
constexpr uint32_t MINUS_LO = 0x80088008u, MINUS_HI = 0x80808080u;   // -8 in the codes' units: rows g, rows g + 8
// A sequence as the split sees it.
struct Seq { int new_, total, p0, pages, tiles; };
__device__ __forceinline__ Seq seq_of(const Attn& p, int s, int rows) {
    const PageSeq x = page_seq(p, s);
    Seq q{x.new_, x.total, 0, 0, 0};
    q.p0 = p.window > 0 ? max(0, x.first - p.window + 1) / XSV_PAGE : 0;
    q.pages = max(1, (x.total + XSV_PAGE - 1) / XSV_PAGE - q.p0);
    const int n_rows = x.new_ * p.group;
    q.tiles = n_rows > p.row_limit ? 0 : (n_rows + rows - 1) / rows;
    return q;
}

// A place in the list of steps: page `pg` of the `q.pages` of (sequence, head, tile).
struct Cursor { int s, head, tile, pg; Seq q; };
__device__ __forceinline__ void advance(const Attn& p, Cursor& c, int rows) {
    if (++c.pg < c.q.pages) return;
    c.pg = 0;
    if (++c.tile < c.q.tiles) return;
    c.tile = 0;
    if (++c.head < p.pool.heads) return;
    c.head = 0;
    while (++c.s < p.n_seqs) {
        c.q = seq_of(p, c.s, rows);
        if (c.q.tiles > 0) return;
    }
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(THREADS, Shape<D, NT>::BLOCKS) page_attn_kernel(const __grid_constant__ Attn p) {
    using R = PageRec<D>;
    constexpr int ROWS = 8 * NT, CT = D / 16, VG = D / 64;
    using S = Shape<D, NT>;
    constexpr int STAGES = S::STAGES;
    // fp16 results are worth two more products a page (see where they are taken); at bf16 their effect, 0.0017 instead of
    // 0.0018 of the result, of which 0.0017 is the output's own rounding, is not
    constexpr bool FINE = std::is_same<T, __half>::value;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) unsigned long long bars[WARPS][STAGES];
    __shared__ int stage_page[WARPS][STAGES];
    __shared__ long long s_base[THREADS + 1], s_warp[WARPS];
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    if (lane < STAGES) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&bars[wid][lane])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    xsv_dep_release();
    xsv_dep_sync();

    // ---- steps of all sequences, scanned: thread i holds `per` consecutive sequences
    const int per = (p.n_seqs + THREADS - 1) / THREADS;
    {
        long long sum = 0;
        for (int s = tid * per; s < min(p.n_seqs, (tid + 1) * per); ++s) {
            const Seq q = seq_of(p, s, ROWS);
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
    }
    __syncthreads();
    const long long steps = s_base[THREADS];
    const int worker = blockIdx.x * WARPS + wid;
    const int workers = (int)min((long long)gridDim.x * WARPS, steps);
    if (lane == 0) p.desc[worker] = make_int4(0, 0, 0, 0);
    if (worker >= workers) return;
    const long long x0 = steps * worker / workers, x1 = steps * (worker + 1) / workers;

    Cursor cur;
    {
        int lo = 0, hi = THREADS - 1;                          // the last thread whose first step is at or before x0
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_base[mid] <= x0) lo = mid; else hi = mid - 1;
        }
        long long at = x0 - s_base[lo];
        cur.s = lo * per;
        for (;; ++cur.s) {
            cur.q = seq_of(p, cur.s, ROWS);
            const long long n = (long long)p.pool.heads * cur.q.tiles * cur.q.pages;
            if (at < n) break;
            at -= n;
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
                if (lane == 0) p.desc[worker] = make_int4(cur.s, cur.head, cur.tile, last - worker + 2);
            }
        }
    }

    uint8_t* ring = smem + wid * S::PER_WARP;
    // query operands: [n][32 channels] of {operand register 0 of both steps, register 1 of both steps}, this lane's
    uint4 q_regs[S::Q_REGS ? NT * (D / 32) : 1] = {};
    uint4* const q_smem = reinterpret_cast<uint4*>(ring + STAGES * R::BYTES) + lane;
    auto query = [&](int i, uint32_t (&q)[2][2]) {
        const uint4 x = S::Q_REGS ? q_regs[S::Q_REGS ? i : 0] : q_smem[i * 32];
        q[0][0] = x.x; q[0][1] = x.y; q[1][0] = x.z; q[1][1] = x.w;
    };
    // Page record of the step at `ld` into stage `st`, then on to the next step, whose page index is fetched already.  The
    // unfilled page's keys are not in its record.
    Cursor ld = cur;
    int ld_left = (int)(x1 - x0), ld_page = -1, ld_part = 0, ld_end = 0;
    const int* ld_row = p.table;
    auto ld_unit = [&]() {                                     // a sequence begins: its table row, the pages there are
        ld_row = p.table + (size_t)min(ld.s, p.n_seqs - 1) * p.width + ld.q.p0;
        ld_part = ld.q.total % XSV_PAGE ? ld.q.total / XSV_PAGE - ld.q.p0 : -1;
        ld_end = ld.s < p.n_seqs ? (ld.q.total + XSV_PAGE - 1) / XSV_PAGE - ld.q.p0 : 0;
    };
    ld_unit();
    if (ld.pg < ld_end) ld_page = ld_row[ld.pg];
    auto issue = [&](int st) {
        if (ld_left == 0) return;
        if (lane == 0) {
            const bool there = (unsigned long long)(long long)ld_page < (unsigned long long)p.pool.n_pages;
            const uint32_t bar = smem_u32(&bars[wid][st]);
            stage_page[wid][st] = there;
            if (there) {
                const uint32_t off = ld.pg == ld_part ? R::V_CODES : 0, bytes = R::BYTES - off;
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(smem_u32(ring + st * R::BYTES + off)), "l"(page_rec<D>(p.pool, ld_page, ld.head) + off), "r"(bytes), "r"(bar) : "memory");
            } else {
                asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
            }
        }
        if (--ld_left > 0) {
            const int seq = ld.s;
            advance(p, ld, ROWS);
            if (ld.s != seq) ld_unit();
            ld_page = ld.pg < ld_end ? ld_row[ld.pg] : -1;
        }
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) issue(i);

    int stage = 0, parity = 0;
    bool failed = false;
    // Refills the stage that was left last, and waits for the one that comes now.
    auto arrive = [&]() {
        __syncwarp();
        if (!failed) {
            issue(stage == 0 ? STAGES - 1 : stage - 1);
            // The warp gives up as one: what follows needs all of its lanes, and near the limit one lane's clock can have run
            // out while another's wait succeeds.
            const uint32_t bar = smem_u32(&bars[wid][stage]);
            if (!__all_sync(0xFFFFFFFFu, mbar_try(bar, parity)) && !__all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity))) {
                failed = true;                                 // nothing is issued any more; what is in flight gets its time
                for (int i = 0; i < STAGES; ++i) mbar_wait_bounded(smem_u32(&bars[wid][(stage + i) % STAGES]), stage + i < STAGES ? parity : parity ^ 1);
                __syncwarp();
            }
        }
        __syncwarp();
    };
    float fac[NT][2], m[NT][2], l[NT][2], zs[NT][2][VG], o[NT][CT][4];
    int qpos[NT][2], pos_lo = 0, pos_hi = 0;
    bool whole = false;                                        // the span holds the unit's first step
    const int n_steps = (int)(x1 - x0);
    for (int at = 0; at < n_steps; ++at) {
        const int head = cur.head, tile = cur.tile;
        if (at == 0 || cur.pg == 0) {
            // ---- a unit begins: its query rows
            whole = cur.pg == 0;
            const int n_rows = cur.q.new_ * p.group, t0 = min(max(p.cu[cur.s], 0), p.n_tokens);
            int first = cur.q.total - cur.q.new_;
            if (cur.q.total == p.width * XSV_PAGE) first = page_seq(p, cur.s).first;      // the sequence may go on beyond its table row
            {
                int i, h;
                page_row(p, tile * ROWS, i, h);
                pos_lo = first + i;
                page_row(p, min(n_rows, tile * ROWS + ROWS) - 1, i, h);
                pos_hi = first + i;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint4 raw[D / 32];
                const int r = tile * ROWS + 8 * n + g;
                float mx = 0.f;
                if (r < n_rows) {
                    int i, h;
                    page_row(p, r, i, h);
                    const T* row = (const T*)p.Q + (size_t)(t0 + i) * p.q_stride + (size_t)(head * p.group + h) * D + 8 * j;
#pragma unroll
                    for (int k = 0; k < D / 32; ++k) raw[k] = *reinterpret_cast<const uint4*>(row + 32 * k);
                } else {
#pragma unroll
                    for (int k = 0; k < D / 32; ++k) raw[k] = make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int k = 0; k < D / 32; ++k)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 f = xsv_unpack2<T>(word(raw[k], w));
                        mx = fmaxf(mx, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
                // exponent that brings the largest element into [2, 4); two factors, since 2^-e alone may leave float32
                const int e = mx > 0.f ? max((__float_as_int(mx) >> 23) - 128, -126) : 0;
                const float s1 = pow2i(-(e / 2)), s2 = pow2i(-(e - e / 2));
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    uint32_t y[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 f = xsv_unpack2<T>(word(raw[k], w));
                        y[w] = pack_h2(f.x * s1 * s2, f.y * s1 * s2);
                    }
                    const uint4 x = make_uint4(y[0], y[2], y[1], y[3]);
                    if (S::Q_REGS) q_regs[S::Q_REGS ? n * (D / 32) + k : 0] = x;
                    else q_smem[(n * (D / 32) + k) * 32] = x;
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
#pragma unroll
                    for (int v = 0; v < VG; ++v) zs[n][c][v] = 0.f;
                }
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[n][c][i] = 0.f;
            }
        }
        // ---- the step's page
        arrive();
        const int pg = cur.q.p0 + cur.pg, tok0 = pg * XSV_PAGE;
        if (stage_page[wid][stage] && !failed) {
            const uint8_t* rec = ring + stage * R::BYTES;
            const bool part = tok0 + XSV_PAGE > cur.q.total;
            const bool mask = tok0 + XSV_PAGE - 1 > pos_lo || part || (p.window > 0 && tok0 <= pos_hi - p.window);
            // logits (in log2 units) are s * f + z, f by row half (i / 2) and column (i % 2)
            float s[NT][4][4], f[NT][4], z[NT][2];
            if (!part) {
                // q . z and, FINE only, what the rounding of q s leaves out (exact) times the middle code, 8, so that the error
                // that stays is that of the codes around their middle
                float qz[NT][3][4];
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    const uint4 sc = *reinterpret_cast<const uint4*>(rec + R::K_SCALE + 64 * k + 16 * j);
                    const uint4 ze = *reinterpret_cast<const uint4*>(rec + R::K_ZERO + 64 * k + 16 * j);
                    uint32_t q[NT][2][2];                          // [operand register][step]
#pragma unroll
                    for (int n = 0; n < NT; ++n) query(n * (D / 32) + k, q[n]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // the offsets as they lie in memory: words 0, 2 on rows g are the first operand register's channels
                            // of both steps, words 1, 3 on rows g + 8 the second's; each product counts on its rows only
                            if (k == 0) mma0(qz[n][h], ze.x, ze.y, ze.z, ze.w, q[n][h][0], q[n][h][1]);
                            else mma(qz[n][h], ze.x, ze.y, ze.z, ze.w, q[n][h][0], q[n][h][1]);
                        }
#pragma unroll
                    for (int kl = 0; kl < 2; ++kl) {
                        const int ks = 2 * k + kl;
                        const uint4 code = *reinterpret_cast<const uint4*>(rec + R::K_CODES + (ks * 32 + lane) * 16);
                        uint32_t b0[NT], b1[NT];
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            b0[n] = hmul2_u(q[n][0][kl], word(sc, 2 * kl));
                            b1[n] = hmul2_u(q[n][1][kl], word(sc, 2 * kl + 1));
                            if (!FINE) continue;
                            const uint32_t e0 = hfnma2_u(q[n][0][kl], word(sc, 2 * kl), b0[n]), e1 = hfnma2_u(q[n][1][kl], word(sc, 2 * kl + 1), b1[n]);
                            if (ks == 0) mma0(qz[n][2], MINUS_EIGHTS, MINUS_EIGHTS, MINUS_EIGHTS, MINUS_EIGHTS, e0, e1);
                            else mma(qz[n][2], MINUS_EIGHTS, MINUS_EIGHTS, MINUS_EIGHTS, MINUS_EIGHTS, e0, e1);
                        }
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint32_t w = word(code, t), v = w >> 8;
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                if (ks == 0) mma0(s[n][t], w & 0x000F000Fu, w & 0x00F000F0u, v & 0x000F000Fu, v & 0x00F000F0u, b0[n], b1[n]);
                                else mma(s[n][t], w & 0x000F000Fu, w & 0x00F000F0u, v & 0x000F000Fu, v & 0x00F000F0u, b0[n], b1[n]);
                            }
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        z[n][c] = (qz[n][0][c] + qz[n][1][c + 2] + (FINE ? qz[n][2][c] : 0.f)) * fac[n][c];
                        f[n][c] = fac[n][c] * 16777216.f;          // 2^24: rows g
                        f[n][c + 2] = fac[n][c] * 1048576.f;       // 2^20: rows g + 8
                    }
                }
            } else {
                const T* tail = tail_rows<T, D>(p.pool, cur.s, pg, head) + (size_t)g * D + 8 * j;
                const int held = cur.q.total - tok0;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[n][t][i] = 0.f;
                    if (16 * t < held) {
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) {
                            const uint4 a = *reinterpret_cast<const uint4*>(tail + (16 * t) * D + 32 * k);
                            const uint4 b = *reinterpret_cast<const uint4*>(tail + (16 * t + 8) * D + 32 * k);
                            uint32_t q[NT][2][2];
#pragma unroll
                            for (int n = 0; n < NT; ++n) query(n * (D / 32) + k, q[n]);
#pragma unroll
                            for (int kl = 0; kl < 2; ++kl)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
                                    mma(s[n][t], to_h2<T>(word(a, 2 * kl)), to_h2<T>(word(b, 2 * kl)), to_h2<T>(word(a, 2 * kl + 1)),
                                        to_h2<T>(word(b, 2 * kl + 1)), q[n][0][kl], q[n][1][kl]);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) { z[n][c] = 0.f; f[n][c] = f[n][c + 2] = fac[n][c]; }
            }
            if (mask) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int tok = tok0 + 16 * t + g + 8 * (i >> 1), at_q = qpos[n][i & 1];
                            const bool seen = tok <= at_q && (p.window <= 0 || tok > at_q - p.window) && tok < cur.q.total;
                            if (!seen) s[n][t][i] = -INFINITY;     // whatever stood there, NaN included
                        }
            }
            // ---- maximum: looked for only when a logit exceeds the one in use
            float xm[NT][2];
            bool raise = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float lo = fmaxf(fmaxf(s[n][0][c], s[n][1][c]), fmaxf(s[n][2][c], s[n][3][c]));
                    const float hi = fmaxf(fmaxf(s[n][0][c + 2], s[n][1][c + 2]), fmaxf(s[n][2][c + 2], s[n][3][c + 2]));
                    xm[n][c] = fmaxf(lo * f[n][c], hi * f[n][c + 2]) + z[n][c];
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
                        for (int v = 0; v < VG; ++v) zs[n][c][v] *= a;
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) { o[n][ct][c] *= a; o[n][ct][c + 2] *= a; }
                    }
            }
            // ---- probabilities, as the products' second operand: tokens 16 t + {2 j, 2 j + 1} (+ 8), row g
            uint32_t b[4][NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float off0 = z[n][0] - m[n][0] + P_BIAS, off1 = z[n][1] - m[n][1] + P_BIAS;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    b[t][n][0] = transpose8(pack_h2(ex2(fmaf(s[n][t][0], f[n][0], off0)), ex2(fmaf(s[n][t][1], f[n][1], off1))));
                    b[t][n][1] = transpose8(pack_h2(ex2(fmaf(s[n][t][2], f[n][2], off0)), ex2(fmaf(s[n][t][3], f[n][3], off1))));
                }
            }
            // ---- its values
#pragma unroll
            for (int v = 0; v < VG; ++v) {
                // scales and offsets of the same tokens, in pairs
                uint32_t sp[8], zp[8], top = 0;
                {
                    const uint8_t* at_s = rec + R::V_SCALE + 128 * v + 32 * j;
                    const uint8_t* at_z = rec + R::V_ZERO + 128 * v + 32 * j;
                    const uint4 s0 = *reinterpret_cast<const uint4*>(at_s), s1 = *reinterpret_cast<const uint4*>(at_s + 16);
                    const uint4 z0 = *reinterpret_cast<const uint4*>(at_z), z1 = *reinterpret_cast<const uint4*>(at_z + 16);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sp[i] = pair_at(s0, s1, i);
                        zp[i] = pair_at(z0, z1, i);
                    }
                }
                if (part) {                                        // places that hold no token: no bits of theirs count
                    asm volatile("" ::: "memory");                 // a branch: as predicated code it would cost every page
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int a = cur.q.total - tok0 - 2 * j - 8 * i;
                        const uint32_t keep = a >= 2 ? 0xFFFFFFFFu : a == 1 ? 0xFFFFu : 0u;
                        sp[i] &= keep;
                        zp[i] &= keep;
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (FINE) zp[i] = hfma2_u(sp[i], EIGHTS, zp[i]);
                    top = __vmaxu2(top, sp[i]);
                }
                // sum of p z (FINE: z + 8 s) on rows g, sum of p on rows g + 8
                float sum[NT][4];
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if (t == 0) mma0(sum[n], zp[0], ONES, zp[1], ONES, b[0][n][0], b[0][n][1]);
                        else mma(sum[n], zp[2 * t], ONES, zp[2 * t + 1], ONES, b[t][n][0], b[t][n][1]);
                    }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        zs[n][c][v] += sum[n][c];
                        if (v == 0) l[n][c] += sum[n][c + 2];
                    }
                // Scales beyond 16, or all below 2^-8, are brought to [8, 16) by a power of two (of their bits: they are positive)
                top = __reduce_max_sync(0xFFFFFFFFu, max(top >> 16, top & 0xFFFFu));
                int e = 0;
                if (top > 0x4C00u || top < 0x1C00u) {
                    e = max((int)(top >> 10) - 18, -15);
                    const uint32_t h = (uint32_t)(15 - e) << 10, down = h | h << 16;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sp[i] = hmul2_u(sp[i], down);
                }
                const float up_lo = pow2i(24 + e), up_hi = pow2i(20 + e);          // back to real units: rows g, rows g + 8
                // Times the value codes.  FINE: around their middle, 8: -8 sum P s, the same for all channels, starts the
                // accumulators (and z + 8 s stands in for z above), so that neither the rounding of P s nor the tensor cores'
                // truncating accumulation sees the codes' mean, which is much larger than what is left of it after sum p z.  For
                // the same reason a page is summed in the tensor cores and the pages in float32 adds, which round (22 000
                // tokens in one accumulator, with the mean, were off by 0.6 %).
                float acc[NT][4][4], mid[NT][4];
                uint32_t ps[4][NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        ps[t][n][0] = hmul2_u(b[t][n][0], sp[2 * t]);
                        ps[t][n][1] = hmul2_u(b[t][n][1], sp[2 * t + 1]);
                        if (!FINE) continue;
                        if (t == 0) mma0(mid[n], MINUS_LO, MINUS_HI, MINUS_LO, MINUS_HI, ps[0][n][0], ps[0][n][1]);
                        else mma(mid[n], MINUS_LO, MINUS_HI, MINUS_LO, MINUS_HI, ps[t][n][0], ps[t][n][1]);
                    }
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint4 code = *reinterpret_cast<const uint4*>(rec + R::V_CODES + ((t * VG + v) * 32 + lane) * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t w = word(code, i), x = w >> 8;
                        const uint32_t a0 = w & 0x000F000Fu, a1 = w & 0x00F000F0u, a2 = x & 0x000F000Fu, a3 = x & 0x00F000F0u;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (t > 0) mma(acc[n][i], a0, a1, a2, a3, ps[t][n][0], ps[t][n][1]);
                            else if (FINE) mma(acc[n][i], a0, a1, a2, a3, ps[0][n][0], ps[0][n][1], mid[n]);
                            else mma0(acc[n][i], a0, a1, a2, a3, ps[0][n][0], ps[0][n][1]);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[n][4 * v + i][c] = fmaf(acc[n][i][c], c < 2 ? up_lo : up_hi, o[n][4 * v + i][c]);
            }
        }
        if (++stage == STAGES) { stage = 0; parity ^= 1; }

        // ---- the unit, or this span's part of it, is done
        const bool ends = cur.pg + 1 == cur.q.pages;
        if (ends || at + 1 == n_steps) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (failed) l[n][c] = NAN;
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        o[n][ct][c] += zs[n][c][ct / 4];
                        o[n][ct][c + 2] += zs[n][c][ct / 4];
                    }
                }
            if (whole && ends) {
                const int n_rows = cur.q.new_ * p.group, t0 = min(max(p.cu[cur.s], 0), p.n_tokens);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int r = tile * ROWS + 8 * n + 2 * j + c;
                        if (r >= n_rows) continue;
                        const int i = p.group_shift >= 0 ? r >> p.group_shift : r / p.group, h = r - i * p.group;
                        const float inv = l[n][c] == 0.f ? 0.f : 1.f / l[n][c];
                        T* dst = (T*)p.out + ((size_t)(t0 + i) * p.q_heads + head * p.group + h) * D + 8 * g;
#pragma unroll
                        for (int v = 0; v < VG; ++v)
                            *reinterpret_cast<uint4*>(dst + 64 * v) = make_uint4(
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
        if (at + 1 < n_steps) advance(p, cur, ROWS);
    }
}

// Units that several warps share.  A block looks at 8 workers' descriptions and merges 16 channels of the units that
// begin to be shared there: its 8 warps take the parts in turn, each lane 4 values (2 rows x 2 channels) of its parts,
// and are merged in the order of the warps.
constexpr int MERGE_WARPS = 8;
template <typename T, int D, int NT>
__global__ void __launch_bounds__(MERGE_WARPS * 32) page_attn_merge_kernel(const __grid_constant__ Attn p, int workers) {
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
    const int w0 = blockIdx.x * 8;
    int4 mine = make_int4(0, 0, 0, 0);
    if (lane < 8 && w0 + lane < workers) mine = p.desc[w0 + lane];
    for (uint32_t todo = __ballot_sync(0xFFFFFFFFu, mine.w > 0); todo; todo &= todo - 1) {     // the same for the whole block
        const int from = __ffs(todo) - 1, w = w0 + from;
        const int4 d = make_int4(__shfl_sync(0xFFFFFFFFu, mine.x, from), __shfl_sync(0xFFFFFFFFu, mine.y, from),
                                 __shfl_sync(0xFFFFFFFFu, mine.z, from), __shfl_sync(0xFFFFFFFFu, mine.w, from));
        Acc acc;
#pragma unroll 4
        for (int i = wid; i < d.w; i += MERGE_WARPS) {
            const float* part = p.part + (size_t)(i == 0 ? 2 * (w - 1) + 1 : 2 * (w + i - 1)) * PF;
            acc.add(reinterpret_cast<const float4*>(part)[(n * CT + ct) * 32 + lane], *reinterpret_cast<const float4*>(part + NT * CT * 128 + 2 * r0));
        }
        const Seq q = seq_of(p, d.x, ROWS);
        const int n_rows = q.new_ * p.group, t0 = min(max(p.cu[d.x], 0), p.n_tokens);
        __syncthreads();                                        // the last unit's reads of the shared arrays
        s_o[wid][lane] = acc.o;
        s_ml[wid][lane] = acc.ml;
        __syncthreads();
        if (wid != 0) continue;
#pragma unroll
        for (int i = 1; i < MERGE_WARPS; ++i) acc.add(s_o[i][lane], s_ml[i][lane]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int r = d.z * ROWS + r0 + c;
            if (r >= n_rows) continue;
            const int i = r / p.group, h = r - i * p.group;
            const float l = c ? acc.ml.w : acc.ml.y, inv = l == 0.f ? 0.f : 1.f / l;
            T* dst = (T*)p.out + ((size_t)(t0 + i) * p.q_heads + d.y * p.group + h) * D + 64 * (ct / 4) + 8 * g + 2 * (ct % 4);
            *reinterpret_cast<uint32_t*>(dst) = page_result2<T>((c ? acc.o.y : acc.o.x) * inv, (c ? acc.o.w : acc.o.z) * inv);
        }
    }
}

// ------------------------------------------------------------------ host side

template <int D, int NT> int workers_at() { return xsv_sm_count() * Shape<D, NT>::BLOCKS * WARPS; }
int workers_of(int head_dim, int nt) {
    return head_dim == 64 ? (nt == 1 ? workers_at<64, 1>() : workers_at<64, 2>()) : (nt == 1 ? workers_at<128, 1>() : workers_at<128, 2>());
}
// 8 query rows a tile where a head has no more, else 16
int tiles_of(int max_new, int group) { return (long long)max_new * group <= 8 ? 1 : 2; }

// Sequences with more query rows a head go to the tensor-memory kernel, whose time does not depend on them up to 128.
// 8 sequences of 8000 tokens, this kernel against that one: 16 heads of 64, 64 rows 100 against 112 us, 80 rows 122
// against 113; 8 key/value heads of 128, 32 rows 52 against 71 us, 48 rows 72 against 71, 64 rows 90 against 71.
int few_rows(int head_dim) { return head_dim == 64 ? 64 : 48; }
bool many_rows(int max_new, int group, int head_dim) { return (long long)max_new * group > few_rows(head_dim); }

size_t workspace_of(int n_tokens, int n_seqs, int max_new, int group, int head_dim) {
    const int nt = tiles_of(max_new, group);
    const size_t workers = (size_t)workers_of(head_dim, nt);
    const size_t pf = (size_t)nt * (head_dim / 16) * 128 + nt * 16;
    const size_t few = align256(workers * sizeof(int4)) + align256(2 * workers * pf * sizeof(float));
    return few + (many_rows(max_new, group, head_dim) ? xsv_page_tc5_workspace(n_tokens, n_seqs, group, head_dim) : 0);
}

template <typename T, int D, int NT> cudaError_t launch(Attn& p, cudaStream_t st) {
    auto kernel = page_attn_kernel<T, D, NT>;
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
    e = xsv_launch_dep(page_attn_merge_kernel<T, D, NT>, dim3((workers + 7) / 8, NT * (D / 16)), dim3(MERGE_WARPS * 32), 0, st, p, workers);
    if (e == cudaSuccess) xsv_count_launch(1);
    return e;
}

template <typename T> cudaError_t launch_any(Attn& p, int head_dim, int nt, cudaStream_t st) {
    if (head_dim == 64) return nt == 1 ? launch<T, 64, 1>(p, st) : launch<T, 64, 2>(p, st);
    return nt == 1 ? launch<T, 128, 1>(p, st) : launch<T, 128, 2>(p, st);
}

}  // namespace

extern "C" size_t xsv_page_attention_workspace(int n_tokens, int n_seqs, int max_new, int q_heads, int kv_heads, int head_dim) {
    if (n_tokens <= 0 || n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS || max_new <= 0) return 0;
    if (kv_heads <= 0 || q_heads < kv_heads || q_heads % kv_heads || (head_dim != 64 && head_dim != 128)) return 0;
    return workspace_of(n_tokens, n_seqs, std::min(max_new, n_tokens), q_heads / kv_heads, head_dim);
}

extern "C" xsv_status xsv_page_attention(const xsv_page_pool* pool, const void* Q, long long q_stride, int n_tokens, int q_heads,
                                         const int* block_table, int table_width, const int* cu_new, const int* total_len,
                                         int n_seqs, int max_new, float scale, int window, void* out, void* workspace,
                                         size_t workspace_bytes, void* stream) {
    return xsv_page_attention_planned(pool, Q, q_stride, n_tokens, q_heads, block_table, table_width, cu_new, total_len, nullptr, n_seqs, max_new, scale,
                                      window, out, workspace, workspace_bytes, stream);
}

extern "C" xsv_status xsv_page_attention_planned(const xsv_page_pool* pool, const void* Q, long long q_stride, int n_tokens, int q_heads,
                                                 const int* block_table, int table_width, const int* cu_new, const int* total_len,
                                                 const int* slot_map, int n_seqs, int max_new, float scale, int window, void* out,
                                                 void* workspace, size_t workspace_bytes, void* stream) {
    Attn p{};
    xsv_status s = xsv_pool_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_tokens < 0 || n_seqs <= 0 || n_seqs > pool->max_seqs || table_width <= 0 || max_new < 0 || window < 0) return XSV_ERR_ARG;
    if (q_heads < pool->kv_heads || q_heads % pool->kv_heads || q_heads > 1 << 16) return XSV_ERR_ARG;
    if (!(scale > 0.f) || !std::isfinite(scale)) return XSV_ERR_ARG;
    if (n_tokens == 0 || max_new == 0) return XSV_OK;
    if (max_new > n_tokens) max_new = n_tokens;
    if (!Q || !block_table || !cu_new || !total_len || !out || !workspace) return XSV_ERR_ARG;
    if (n_tokens > 1 && q_stride < (long long)q_heads * pool->head_dim) return XSV_ERR_ARG;
    if (((uintptr_t)Q | (uintptr_t)out | (uintptr_t)workspace) & 15 || q_stride & 7) return XSV_ERR_SHAPE;
    const int group = q_heads / pool->kv_heads, nt = tiles_of(max_new, group);
    // rows of a sequence and its tokens are 32-bit numbers
    if ((long long)n_tokens * group > 1LL << 30 || (long long)table_width * XSV_PAGE > 1LL << 30) return XSV_ERR_LIMIT;
    if (workspace_bytes < workspace_of(n_tokens, n_seqs, max_new, group, pool->head_dim)) return XSV_ERR_ARG;
    p.Q = Q; p.out = out; p.table = block_table; p.cu = cu_new; p.total = total_len; p.slot = slot_map; p.q_stride = q_stride;
    const size_t workers = (size_t)workers_of(pool->head_dim, nt), pf = (size_t)nt * (pool->head_dim / 16) * 128 + nt * 16;
    p.desc = (int4*)workspace;
    p.part = (float*)((char*)workspace + align256(workers * sizeof(int4)));
    void* const more = (char*)p.part + align256(2 * workers * pf * sizeof(float));
    p.scale = scale * 1.4426950408889634f;
    p.width = table_width; p.n_seqs = n_seqs; p.n_tokens = n_tokens; p.q_heads = q_heads; p.group = group;
    p.window = window;
    p.group_shift = -1;
    for (int b = 0; b < 16; ++b) if (group == 1 << b) p.group_shift = b;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    p.row_limit = 1 << 30;
    if (many_rows(max_new, group, pool->head_dim)) {
        p.row_limit = n_seqs == 1 ? 0 : few_rows(pool->head_dim);
        e = xsv_launch_page_tc5(p, pool->dtype, pool->head_dim, more, st);
    }
    if (e == cudaSuccess && p.row_limit > 0)
        e = pool->dtype == XSV_F16 ? launch_any<__half>(p, pool->head_dim, nt, st) : launch_any<__nv_bfloat16>(p, pool->head_dim, nt, st);
    return e == cudaSuccess ? XSV_OK : xsv_cuda_status(e);
}
