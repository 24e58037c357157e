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
// and elements below 2^-14 lose at most 2^-25 absolutely.  P s is scaled by a running power of two per warp (like the
// running maximum) so that it uses fp16's range whatever the values' magnitude.  Rounding q s, P s and the result
// to fp16 / the output type are the only roundings below float32; sums, maxima and the output accumulate in float32.
//
// Work split.  A unit is (sequence, key/value head, tile of 8 NT query rows); its pages are the steps.  All steps of all
// units are dealt in equal contiguous spans to the warps of the grid, so ragged lengths and few sequences fill the GPU
// alike; a warp works alone (own ring of page records in shared memory, filled by bulk copies, own softmax state), no
// block-wide barrier in the loop.  A unit shared by several warps is merged by a second kernel in the order of the
// warps, so results do not depend on timing.  Each block finds its spans itself by scanning the lengths.
#include <algorithm>
#include <cmath>

#include "../../include/xsv.h"
#include "page_layout.cuh"
#include "xsv_kernels.h"

namespace {

constexpr int WARPS = 4, THREADS = WARPS * 32;
constexpr unsigned long long WAIT_LIMIT_NS = 2000000000ull;

struct Attn {
    PoolView pool;
    const void* Q;
    void* out;
    const int* table;
    const int* cu;
    const int* total;
    int4* desc;          // [workers] units that are shared: {sequence, unit in it, parts, -}; parts 0: none starts here
    float* part;         // [2 workers][slot] unnormalised rows
    long long q_stride;
    float scale;         // times log2 e
    int width, n_seqs, n_tokens, q_heads, group, max_new, window;
    int group_shift;     // log2 of group where it is a power of two, else -1
};

// one unnormalised tile: [NT][D / 16][32 lanes] float4, then maxima and sums [8 NT] float2
template <int D, int NT> struct Part { static constexpr int FLOATS = NT * (D / 16) * 128 + NT * 16; };

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ unsigned long long globaltimer() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded: false once the limit has passed.
__device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity) {
    const unsigned long long t0 = globaltimer();
    while (globaltimer() - t0 < WAIT_LIMIT_NS)
        if (mbar_try(bar, parity)) return true;
    return false;
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_h2(float a, float b) {   // saturating
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <typename T> __device__ __forceinline__ uint32_t to_h2(uint32_t w);
template <> __device__ __forceinline__ uint32_t to_h2<__half>(uint32_t w) { return w; }
template <> __device__ __forceinline__ uint32_t to_h2<__nv_bfloat16>(uint32_t w) {
    return pack_h2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ uint32_t hmul2_u(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ float half_at(const uint4& v, int i) {
    const uint32_t w = word(v, i >> 1);
    return __half2float(__ushort_as_half((unsigned short)(i & 1 ? w >> 16 : w & 0xFFFFu)));
}
__device__ __forceinline__ float pow2i(int e) {            // 2^e, clamped to what float32 holds as a normal number
    return __int_as_float((min(max(e, -126), 127) + 127) << 23);
}

// A sequence as the split sees it.
struct Seq { int new_, total, p0, pages, units; };
__device__ __forceinline__ Seq seq_of(const Attn& p, int s, int rows) {
    Seq q;
    const int a = min(max(p.cu[s], 0), p.n_tokens), b = min(max(p.cu[s + 1], a), p.n_tokens);
    q.new_ = min(b - a, p.max_new);
    q.total = (int)min((long long)max(p.total[s], 0), (long long)p.width * XSV_PAGE);
    const int first = q.total - q.new_;                       // position of the first new token
    q.p0 = p.window > 0 ? max(0, first - p.window + 1) / XSV_PAGE : 0;
    q.pages = max(1, (q.total + XSV_PAGE - 1) / XSV_PAGE - q.p0);
    q.units = q.new_ > 0 ? p.pool.heads * ((q.new_ * p.group + rows - 1) / rows) : 0;
    return q;
}

// A place in the list of steps: unit `u` of sequence `s`, page `p` of its `q.pages`.
struct Cursor { int s, u, pg; Seq q; };
__device__ __forceinline__ void advance(const Attn& p, Cursor& c, int rows) {
    if (++c.pg < c.q.pages) return;
    c.pg = 0;
    if (++c.u < c.q.units) return;
    c.u = 0;
    while (++c.s < p.n_seqs) {
        c.q = seq_of(p, c.s, rows);
        if (c.q.units > 0) return;
    }
}

template <typename T, int D, int NT, int STAGES>
__global__ void __launch_bounds__(THREADS) page_attn_kernel(const __grid_constant__ Attn p) {
    using R = PageRec<D>;
    constexpr int ROWS = 8 * NT, KS = D / 16, CT = D / 16, VG = D / 64;
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
            sum += (long long)q.units * q.pages;
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
            const long long n = (long long)cur.q.units * cur.q.pages;
            if (at < n) break;
            at -= n;
        }
        cur.u = (int)(at / cur.q.pages);
        cur.pg = (int)(at % cur.q.pages);
        // The first worker that continues a unit describes how many parts it has.
        if (cur.pg > 0) {
            const long long unit0 = x0 - cur.pg, unit1 = unit0 + cur.q.pages;
            if (steps * (worker - 1) / workers <= unit0) {
                int last = worker;                             // the worker of the unit's last step
                long long k = (unit1 - 1) * workers / steps;
                if (k > last) last = (int)k;
                while (last + 1 < workers && steps * (last + 1) / workers < unit1) ++last;
                while (last > worker && steps * last / workers >= unit1) --last;
                if (lane == 0) p.desc[worker] = make_int4(cur.s, cur.u, last - worker + 2, 0);
            }
        }
    }

    uint8_t* ring = smem + wid * STAGES * R::BYTES;
    // Page record of the step at `c` into stage `st`.  The unfilled page's keys are not in the record.
    Cursor ld = cur;
    long long ld_at = x0;
    auto table_at = [&](const Cursor& c) {
        const int pg = c.q.p0 + c.pg;
        int id = -1;
        if (c.s < p.n_seqs && c.s < p.pool.max_seqs && pg < p.width && pg * XSV_PAGE < c.q.total) id = p.table[(size_t)c.s * p.width + pg];
        return id >= 0 && id < p.pool.n_pages ? id : -1;
    };
    int ld_page = table_at(ld);
    auto issue = [&](int st) {                                 // loads the step at `ld` and advances it
        if (ld_at >= x1) return;
        const int tiles = ld.q.units / p.pool.heads, head = ld.u / tiles;
        if (lane == 0) {
            stage_page[wid][st] = ld_page;
            if (ld_page >= 0) {
                const uint8_t* rec = page_rec<D>(p.pool, ld_page, head);
                const bool part = (ld.q.p0 + ld.pg + 1) * XSV_PAGE > ld.q.total;
                const uint32_t off = part ? R::V_CODES : 0, bytes = R::BYTES - off, bar = smem_u32(&bars[wid][st]);
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(smem_u32(ring + st * R::BYTES + off)), "l"(rec + off), "r"(bytes), "r"(bar) : "memory");
            } else {
                asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&bars[wid][st])) : "memory");
            }
        }
        ++ld_at;
        if (ld_at < x1) {
            advance(p, ld, ROWS);
            ld_page = table_at(ld);
        }
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) issue(i);

    int stage = 0, parity = 0;
    bool failed = false;
    uint32_t qf[NT][KS][2];
    float fac[NT][2], m[NT][2], l[NT][2], zs[NT][2][VG], o[NT][CT][4];
    int qpos[NT][2], e_run = 0, pos_lo = 0, pos_hi = 0;
    bool fresh = true;                                         // no page of the unit yet: e_run is not set
    bool whole = false;                                        // the span holds the unit's first step
    for (long long at = x0; at < x1; ++at) {
        const int tiles = cur.q.units / p.pool.heads, head = cur.u / tiles, tile = cur.u - head * tiles;
        if (at == x0 || cur.pg == 0) {
            // ---- a unit begins: its query rows
            whole = cur.pg == 0;
            fresh = true;
            const int n_rows = cur.q.new_ * p.group, t0 = min(max(p.cu[cur.s], 0), p.n_tokens), first = cur.q.total - cur.q.new_;
            auto split = [&](int r, int& i, int& h) {
                i = p.group_shift >= 0 ? r >> p.group_shift : r / p.group;
                h = r - i * p.group;
            };
            {
                int i, h;
                split(tile * ROWS, i, h);
                pos_lo = first + i;
                split(min(n_rows, tile * ROWS + ROWS) - 1, i, h);
                pos_hi = first + i;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint4 raw[D / 32];
                const int r = tile * ROWS + 8 * n + g;
                float mx = 0.f;
                if (r < n_rows) {
                    int i, h;
                    split(r, i, h);
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
                for (int k = 0; k < D / 32; ++k)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 f = xsv_unpack2<T>(word(raw[k], w));
                        qf[n][2 * k + (w >> 1)][w & 1] = pack_h2(f.x * s1 * s2, f.y * s1 * s2);
                    }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int er = __shfl_sync(0xFFFFFFFFu, e, 4 * (2 * j + c));
                    fac[n][c] = p.scale * pow2i(er);
                    const int row = tile * ROWS + 8 * n + 2 * j + c;
                    int i, h;
                    split(row, i, h);
                    qpos[n][c] = row < n_rows ? first + i : -1;
                    m[n][c] = -INFINITY;
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
        __syncwarp();
        if (!failed) {
            issue(stage == 0 ? STAGES - 1 : stage - 1);        // the stage that the last step left
            if (!mbar_try(smem_u32(&bars[wid][stage]), parity) && !mbar_wait_slow(smem_u32(&bars[wid][stage]), parity)) {
                failed = true;                                 // nothing is issued any more; what is in flight gets its time
                for (int i = 0; i < STAGES; ++i) mbar_wait_slow(smem_u32(&bars[wid][(stage + i) % STAGES]), stage + i < STAGES ? parity : parity ^ 1);
            }
        }
        __syncwarp();
        const uint8_t* rec = ring + stage * R::BYTES;
        const int page = stage_page[wid][stage], pg = cur.q.p0 + cur.pg, tok0 = pg * XSV_PAGE;
        if (page >= 0 && !failed) {
            const bool part = tok0 + XSV_PAGE > cur.q.total;
            const bool mask = tok0 + XSV_PAGE - 1 > pos_lo || part || (p.window > 0 && tok0 <= pos_hi - p.window);
            float s[NT][4][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][t][i] = 0.f;
            if (!part) {
                float qz[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) qz[n][i] = 0.f;
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    const uint4 sc = *reinterpret_cast<const uint4*>(rec + R::K_SCALE + 64 * k + 16 * j);
                    const uint4 ze = *reinterpret_cast<const uint4*>(rec + R::K_ZERO + 64 * k + 16 * j);
#pragma unroll
                    for (int kl = 0; kl < 2; ++kl) {
                        const int ks = 2 * k + kl;
                        const uint4 code = *reinterpret_cast<const uint4*>(rec + R::K_CODES + (ks * 32 + lane) * 16);
                        uint32_t b0[NT], b1[NT];
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            b0[n] = hmul2_u(qf[n][ks][0], word(sc, 2 * kl));
                            b1[n] = hmul2_u(qf[n][ks][1], word(sc, 2 * kl + 1));
                            mma(qz[n], word(ze, 2 * kl), word(ze, 2 * kl), word(ze, 2 * kl + 1), word(ze, 2 * kl + 1), qf[n][ks][0], qf[n][ks][1]);
                        }
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint32_t w = word(code, t), v = w >> 8;
#pragma unroll
                            for (int n = 0; n < NT; ++n)
                                mma(s[n][t], w & 0x000F000Fu, w & 0x00F000F0u, v & 0x000F000Fu, v & 0x00F000F0u, b0[n], b1[n]);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float z0 = qz[n][0] * fac[n][0], z1 = qz[n][1] * fac[n][1];
                    const float lo0 = fac[n][0] * 16777216.f, lo1 = fac[n][1] * 16777216.f;      // 2^24: row g
                    const float hi0 = fac[n][0] * 1048576.f, hi1 = fac[n][1] * 1048576.f;        // 2^20: row g + 8
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        s[n][t][0] = fmaf(s[n][t][0], lo0, z0);
                        s[n][t][1] = fmaf(s[n][t][1], lo1, z1);
                        s[n][t][2] = fmaf(s[n][t][2], hi0, z0);
                        s[n][t][3] = fmaf(s[n][t][3], hi1, z1);
                    }
                }
            } else {
                const T* tail = tail_rows<T, D>(p.pool, cur.s, pg, head) + (size_t)g * D + 8 * j;
                const int held = cur.q.total - tok0;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (16 * t < held) {
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) {
                            const uint4 a = *reinterpret_cast<const uint4*>(tail + (16 * t) * D + 32 * k);
                            const uint4 b = *reinterpret_cast<const uint4*>(tail + (16 * t + 8) * D + 32 * k);
#pragma unroll
                            for (int kl = 0; kl < 2; ++kl)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
                                    mma(s[n][t], to_h2<T>(word(a, 2 * kl)), to_h2<T>(word(b, 2 * kl)), to_h2<T>(word(a, 2 * kl + 1)),
                                        to_h2<T>(word(b, 2 * kl + 1)), qf[n][2 * k + kl][0], qf[n][2 * k + kl][1]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[n][t][i] *= fac[n][i & 1];
                }
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
            // ---- value parameters of the lane's tokens 8 i + g; the running power of two
            uint4 vsc[VG], vze[VG];
            uint32_t top = 0;
#pragma unroll
            for (int v = 0; v < VG; ++v) {
                vsc[v] = *reinterpret_cast<const uint4*>(rec + R::V_SCALE + 128 * v + 16 * g);
                vze[v] = *reinterpret_cast<const uint4*>(rec + R::V_ZERO + 128 * v + 16 * g);
                if (part) {                                        // places that hold no token: no bits of theirs count
                    uint32_t keep[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int a = tok0 + 16 * i + g;
                        keep[i] = (a < cur.q.total ? 0xFFFFu : 0u) | (a + 8 < cur.q.total ? 0xFFFF0000u : 0u);
                    }
                    vsc[v] = make_uint4(vsc[v].x & keep[0], vsc[v].y & keep[1], vsc[v].z & keep[2], vsc[v].w & keep[3]);
                    vze[v] = make_uint4(vze[v].x & keep[0], vze[v].y & keep[1], vze[v].z & keep[2], vze[v].w & keep[3]);
                }
                top = __vmaxu2(top, __vmaxu2(__vmaxu2(vsc[v].x, vsc[v].y), __vmaxu2(vsc[v].z, vsc[v].w)));
            }
            top = max(top >> 16, top & 0xFFFFu);                   // scales are positive: their order is that of their bits
            top = __reduce_max_sync(0xFFFFFFFFu, top);
            // exponent of the largest scale (fp16 bits; 2^(field - 15), subnormals counted as 2^-14): P s <= 2^14
            const int e_page = (int)(max(top, 0x0400u) >> 10) - 15 - 13;
            bool raise = fresh || e_page > e_run;
            // ---- running maximum
            float mn[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = fmaxf(fmaxf(fmaxf(s[n][0][c], s[n][0][c + 2]), fmaxf(s[n][1][c], s[n][1][c + 2])),
                                    fmaxf(fmaxf(s[n][2][c], s[n][2][c + 2]), fmaxf(s[n][3][c], s[n][3][c + 2])));
                    x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 16));
                    mn[n][c] = fmaxf(m[n][c], x);
                    raise = raise || mn[n][c] > m[n][c];
                }
            if (__any_sync(0xFFFFFFFFu, raise)) {
                const int e_new = fresh ? e_page : max(e_run, e_page);
                const float down = fresh ? 1.f : pow2i(e_run - e_new);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float a = m[n][c] == -INFINITY ? 0.f : ex2(m[n][c] - mn[n][c]);
                        m[n][c] = mn[n][c];
                        l[n][c] *= a;
#pragma unroll
                        for (int v = 0; v < VG; ++v) zs[n][c][v] *= a;
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) { o[n][ct][c] *= a * down; o[n][ct][c + 2] *= a * down; }
                    }
                e_run = e_new;
                fresh = false;
            }
            const float unit = pow2i(-e_run);
            // ---- probabilities, scaled by the tokens' value scales, and the product with the value codes
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                float sc[VG][2], ze[VG][2];
#pragma unroll
                for (int v = 0; v < VG; ++v)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        sc[v][h] = half_at(vsc[v], 2 * t + h) * unit;
                        ze[v][h] = half_at(vze[v], 2 * t + h);
                    }
                uint32_t b[NT][VG][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float pr[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float mc = m[n][i & 1];
                        pr[i] = ex2(s[n][t][i] - (mc == -INFINITY ? 0.f : mc));
                    }
                    l[n][0] += pr[0] + pr[2];
                    l[n][1] += pr[1] + pr[3];
#pragma unroll
                    for (int v = 0; v < VG; ++v) {
                        zs[n][0][v] = fmaf(pr[0], ze[v][0], fmaf(pr[2], ze[v][1], zs[n][0][v]));
                        zs[n][1][v] = fmaf(pr[1], ze[v][0], fmaf(pr[3], ze[v][1], zs[n][1][v]));
                        b[n][v][0] = transpose8(pack_h2(pr[0] * sc[v][0], pr[1] * sc[v][0]));
                        b[n][v][1] = transpose8(pack_h2(pr[2] * sc[v][1], pr[3] * sc[v][1]));
                    }
                }
#pragma unroll
                for (int v = 0; v < VG; ++v) {
                    const uint4 code = *reinterpret_cast<const uint4*>(rec + R::V_CODES + ((t * VG + v) * 32 + lane) * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t w = word(code, i), x = w >> 8;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            mma(o[n][4 * v + i], w & 0x000F000Fu, w & 0x00F000F0u, x & 0x000F000Fu, x & 0x00F000F0u, b[n][v][0], b[n][v][1]);
                    }
                }
            }
        }
        if (++stage == STAGES) { stage = 0; parity ^= 1; }

        // ---- the unit, or this span's part of it, is done
        const bool ends = cur.pg + 1 == cur.q.pages;
        if (ends || at + 1 == x1) {
            const float up = fresh ? 0.f : pow2i(e_run);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) {
                        l[n][c] += __shfl_xor_sync(0xFFFFFFFFu, l[n][c], x);
#pragma unroll
                        for (int v = 0; v < VG; ++v) zs[n][c][v] += __shfl_xor_sync(0xFFFFFFFFu, zs[n][c][v], x);
                    }
                    if (failed) l[n][c] = NAN;
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        o[n][ct][c] = fmaf(o[n][ct][c] * 16777216.f, up, zs[n][c][ct / 4]);
                        o[n][ct][c + 2] = fmaf(o[n][ct][c + 2] * 1048576.f, up, zs[n][c][ct / 4]);
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
                                xsv_pack2<T>(o[n][4 * v][c] * inv, o[n][4 * v][c + 2] * inv), xsv_pack2<T>(o[n][4 * v + 1][c] * inv, o[n][4 * v + 1][c + 2] * inv),
                                xsv_pack2<T>(o[n][4 * v + 2][c] * inv, o[n][4 * v + 2][c + 2] * inv), xsv_pack2<T>(o[n][4 * v + 3][c] * inv, o[n][4 * v + 3][c + 2] * inv));
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
        if (at + 1 < x1) advance(p, cur, ROWS);
    }
}

// Units that several warps share: parts in the order of the warps, one block per unit; a thread merges 4 values
// (2 rows x 2 channels) over all parts.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(NT * D * 2) page_attn_merge_kernel(const __grid_constant__ Attn p) {
    constexpr int ROWS = 8 * NT, CT = D / 16, PF = Part<D, NT>::FLOATS;
    __shared__ float s_max[ROWS];
    xsv_dep_release();
    xsv_dep_sync();
    const int w = blockIdx.x + 1;
    const int4 d = p.desc[w];
    if (d.z == 0) return;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    auto part = [&](int i) { return p.part + (size_t)(i == 0 ? 2 * (w - 1) + 1 : 2 * (w + i - 1)) * PF; };
    auto stats = [&](int i, int r) { return reinterpret_cast<const float2*>(part(i) + NT * CT * 128)[r]; };
    for (int r = wid; r < ROWS; r += NT * D * 2 / 32) {
        float mx = -INFINITY;
        for (int i = lane; i < d.z; i += 32) mx = fmaxf(mx, stats(i, r).x);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
        if (lane == 0) s_max[r] = mx == -INFINITY ? 0.f : mx;
    }
    __syncthreads();
    const Seq q = seq_of(p, d.x, ROWS);
    const int tiles = q.units / p.pool.heads, head = d.y / tiles, tile = d.y - head * tiles;
    const int n = tid / (CT * 32), ct = tid / 32 % CT, g = lane >> 2, j = lane & 3, r0 = 8 * n + 2 * j;
    const float m0 = s_max[r0], m1 = s_max[r0 + 1];
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float l0 = 0.f, l1 = 0.f;
#pragma unroll 4
    for (int i = 0; i < d.z; ++i) {
        const float4 x = reinterpret_cast<const float4*>(part(i))[tid];
        const float4 ml = *reinterpret_cast<const float4*>(part(i) + NT * CT * 128 + 2 * r0);
        const float a = ex2(ml.x - m0), b = ex2(ml.z - m1);
        o.x = fmaf(x.x, a, o.x); o.y = fmaf(x.y, b, o.y); o.z = fmaf(x.z, a, o.z); o.w = fmaf(x.w, b, o.w);
        l0 = fmaf(ml.y, a, l0); l1 = fmaf(ml.w, b, l1);
    }
    const int n_rows = q.new_ * p.group, t0 = min(max(p.cu[d.x], 0), p.n_tokens);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int r = tile * ROWS + r0 + c;
        if (r >= n_rows) continue;
        const int i = r / p.group, h = r - i * p.group;
        const float l = c ? l1 : l0, inv = l == 0.f ? 0.f : 1.f / l;
        T* dst = (T*)p.out + ((size_t)(t0 + i) * p.q_heads + head * p.group + h) * D + 64 * (ct / 4) + 8 * g + 2 * (ct % 4);
        *reinterpret_cast<uint32_t*>(dst) = xsv_pack2<T>((c ? o.y : o.x) * inv, (c ? o.w : o.z) * inv);
    }
}

// ------------------------------------------------------------------ host side
template <int D> constexpr int stages() { return 3; }
template <int D> constexpr int blocks_per_sm() { return D == 64 ? 4 : 2; }
template <int D> constexpr size_t ring_bytes() { return (size_t)WARPS * stages<D>() * PageRec<D>::BYTES; }
constexpr size_t align256(size_t v) { return (v + 255) / 256 * 256; }

int grid_of(int head_dim) { return xsv_sm_count() * (head_dim == 64 ? blocks_per_sm<64>() : blocks_per_sm<128>()); }
// 8 query rows a tile where a head has no more, else 16
int tiles_of(int max_new, int group) { return (long long)max_new * group <= 8 ? 1 : 2; }

size_t workspace_of(int head_dim, int nt) {
    const size_t workers = (size_t)grid_of(head_dim) * WARPS;
    const size_t pf = (size_t)nt * (head_dim / 16) * 128 + nt * 16;
    return align256(workers * sizeof(int4)) + 2 * workers * pf * sizeof(float);
}

template <typename T, int D, int NT> cudaError_t launch(Attn& p, cudaStream_t st) {
    auto kernel = page_attn_kernel<T, D, NT, stages<D>()>;
    constexpr size_t smem = ring_bytes<D>();
    static XsvPerDeviceInt ready;
    const int dev = xsv_current_device();
    if (!ready.get(dev)) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        ready.set(dev, 1);
    }
    const int grid = grid_of(D);
    cudaError_t e = xsv_launch_dep(kernel, dim3(grid), dim3(THREADS), smem, st, p);
    if (e != cudaSuccess) return e;
    xsv_count_launch(1);
    e = xsv_launch_dep(page_attn_merge_kernel<T, D, NT>, dim3(grid * WARPS - 1), dim3(NT * D * 2), 0, st, p);
    if (e == cudaSuccess) xsv_count_launch(1);
    return e;
}

template <typename T> cudaError_t launch_any(Attn& p, int head_dim, int nt, cudaStream_t st) {
    if (head_dim == 64) return nt == 1 ? launch<T, 64, 1>(p, st) : launch<T, 64, 2>(p, st);
    return nt == 1 ? launch<T, 128, 1>(p, st) : launch<T, 128, 2>(p, st);
}

}  // namespace

extern "C" size_t xsv_page_attention_workspace(int n_seqs, int max_new, int q_heads, int kv_heads, int head_dim) {
    if (n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS || max_new <= 0 || kv_heads <= 0 || q_heads < kv_heads || q_heads % kv_heads) return 0;
    if (head_dim != 64 && head_dim != 128) return 0;
    return workspace_of(head_dim, tiles_of(max_new, q_heads / kv_heads));
}

extern "C" xsv_status xsv_page_attention(const xsv_page_pool* pool, const void* Q, long long q_stride, int n_tokens, int q_heads,
                                         const int* block_table, int table_width, const int* cu_new, const int* total_len,
                                         int n_seqs, int max_new, float scale, int window, void* out, void* workspace,
                                         size_t workspace_bytes, void* stream) {
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
    if ((long long)max_new * group > 1LL << 30 || (long long)table_width * XSV_PAGE > 1LL << 30) return XSV_ERR_LIMIT;
    if (workspace_bytes < workspace_of(pool->head_dim, nt)) return XSV_ERR_ARG;
    p.Q = Q; p.out = out; p.table = block_table; p.cu = cu_new; p.total = total_len; p.q_stride = q_stride;
    p.desc = (int4*)workspace;
    p.part = (float*)((char*)workspace + align256((size_t)grid_of(pool->head_dim) * WARPS * sizeof(int4)));
    p.scale = scale * 1.4426950408889634f;
    p.width = table_width; p.n_seqs = n_seqs; p.n_tokens = n_tokens; p.q_heads = q_heads; p.group = group; p.max_new = max_new;
    p.window = window;
    p.group_shift = -1;
    for (int b = 0; b < 16; ++b) if (group == 1 << b) p.group_shift = b;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = pool->dtype == XSV_F16 ? launch_any<__half>(p, pool->head_dim, nt, st) : launch_any<__nv_bfloat16>(p, pool->head_dim, nt, st);
    return e == cudaSuccess ? XSV_OK : xsv_cuda_status(e);
}
