// Writing the 8-bit pages of the shared pool, and reading them back as values.
//
// xsv_page8_append: codes are written as their tokens come, without a 16-bit copy that waits for the page to fill: the block's
// scale is a power of two, so that a later token with a larger magnitude raises it and the codes that stand there are moved to
// the new scale (exact unless they become subnormal).  A page's new rows are read once, their largest magnitude is found, and they are
// stored as codes: by a warp where they are few, else by a block, keys and values apart.  Whoever brings a page's last token also sums
// its key codes per channel, exactly (at most 64 * 448, in steps of 2^-9: 24 bits, so that no order of summation matters), for the
// mean key that a selection scores.
// Bound by HBM for prompts, 2 bytes read and 1 written per element, and by latency for single tokens: five loads that wait for one another.
// What counts is warps in flight (36 a multiprocessor at head_dim 64, 28 at 128, against 20: 14.5 against 18.7 us) and a lane's 8
// channels, whose codes fill whole sectors of both records' orders (16 channels: 21.7).
//
// xsv_page8_read: a thread looks one token up and decodes 8 channels of it, of up to 4 heads.
//
// Measured.  Append of 19 735 prompt tokens, 8 heads of 64, fp16: 14.5 us, 4.2 TB/s; 8 heads of 128, bf16: 24.5 us, 4.95 TB/s; one token for each
// of 256 sequences, 8 heads of 128: 4.3 us.  Reading 19 735 tokens of 8 x 64 back: 12.8 us, 4.7 TB/s; 8150 of 8 x 128: 11.2 us, 4.5 TB/s.
// From 4000 to 158 000 tokens both are a fixed part (launch, dependent lookups) and a rate: append 2.9 us and 5.4 TB/s at heads of 64, 3.6 us and the
// copy rate at 128; read 2.2 us and 6.1 TB/s, 2.9 us and 6.3 TB/s.
#include <type_traits>

#include "../../include/xsv.h"
#include "page8_layout.cuh"
#include "xsv_kernels.h"

namespace {

struct Append8 {
    PoolView pool;
    const void* K;
    const void* V;
    long long k_stride, v_stride;
    const int* slot;
    const int* seq;
    const int* cu;
    const int* total;
    int n_tokens, n_seqs;
    int few_blocks, across;            // blocks that store a few tokens of a page; heads of each of the others
};
__device__ __forceinline__ bool place_of(const Append8& p, int t, PagePlace& q) {
    return page_place(p.slot, p.seq, p.cu, p.total, p.n_tokens, p.n_seqs, p.pool.n_pages, t, q);
}

// Inputs count as at most 65504 in magnitude (bf16: 65536, whose code is the same).  Where a magnitude, as bits, is beyond BOUND,
// infinities and NaN among them, pairs are brought to it; a NaN becomes the bound.
template <typename T> constexpr uint32_t BOUND = 0x7BFFu;
template <> constexpr uint32_t BOUND<__nv_bfloat16> = 0x4780u;
template <typename T> __device__ __forceinline__ uint32_t bounded2(uint32_t w) {
    constexpr uint32_t HI = BOUND<T> * 0x10001u, LO = HI | 0x80008000u;
    return max2<T>(min2<T>(w, HI), LO);
}
template <typename T> __device__ __forceinline__ uint4 bounded8(const uint4& r) { return make_uint4(bounded2<T>(r.x), bounded2<T>(r.y), bounded2<T>(r.z), bounded2<T>(r.w)); }
// 8 channels of a row, and the larger of the magnitudes so far (as bit patterns, two a word: positive 16-bit floats compare
// like whole numbers).
__device__ __forceinline__ uint4 load8(const void* x) { return *reinterpret_cast<const uint4*>(x); }
__device__ __forceinline__ uint32_t mag8(const uint4& r, uint32_t m) {
    constexpr uint32_t ABS = 0x7FFF7FFFu;
    return __vmaxu2(m, __vmaxu2(__vmaxu2(r.x & ABS, r.y & ABS), __vmaxu2(r.z & ABS, r.w & ABS)));
}
__device__ __forceinline__ uint32_t warp_mag(uint32_t m) { return __reduce_max_sync(0xFFFFFFFFu, max(m & 0xFFFFu, m >> 16)); }
template <typename T> __device__ __forceinline__ int exponent_of_mag(uint32_t m) { return p8_exponent(xsv_unpack2<T>(min(m, BOUND<T>)).x); }

// Codes of 8 channels for the scale 2^e.  x / 2^e is taken in the inputs' own type: exact, or so small that its code is 0.  fp16
// does not hold 2^-e for e below -14: by way of float32 then.
template <typename T> struct Quant;
template <> struct Quant<__nv_bfloat16> {
    uint32_t inv;
    __device__ __forceinline__ explicit Quant(int e) : inv((uint32_t)(127 - e) << 7) { inv |= inv << 16; }
    __device__ __forceinline__ uint32_t two(uint32_t w) const {
        uint32_t y;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(w), "r"(inv));
        const float2 f = xsv_unpack2<__nv_bfloat16>(y);
        return p8_codes2(f.x, f.y);
    }
};
template <> struct Quant<__half> {
    uint32_t inv;
    float wide;                                                // 0: inv holds it
    __device__ __forceinline__ explicit Quant(int e) : inv((uint32_t)(15 - max(e, -14)) << 10), wide(e < -14 ? p8_pow2(-e) : 0.f) { inv |= inv << 16; }
    __device__ __forceinline__ uint32_t two(uint32_t w) const {
        if (wide != 0.f) {                                     // the same for the whole warp
            const float2 f = xsv_unpack2<__half>(w);
            return p8_codes2(f.x * wide, f.y * wide);
        }
        uint32_t y;
        unsigned short r;
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(w), "r"(inv));
        asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(y));
        return r;
    }
};
template <typename T> __device__ __forceinline__ uint2 codes8(const uint4& r, const Quant<T>& q) {
    return make_uint2(__byte_perm(q.two(r.x), q.two(r.y), 0x5410), __byte_perm(q.two(r.z), q.two(r.w), 0x5410));
}
// four codes at another scale
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
    uint32_t lo, hi;
    p8_halves(w, lo, hi);
    const float2 a = xsv_unpack2<__half>(lo), b = xsv_unpack2<__half>(hi);
    return p8_codes2(a.x * f, a.y * f) | p8_codes2(b.x * f, b.y * f) << 16;
}
__device__ __forceinline__ uint2 rescale8(const uint2& w, float f) { return make_uint2(rescale4(w.x, f), rescale4(w.y, f)); }
__device__ __forceinline__ void add4(uint32_t w, float* s) {
    uint32_t lo, hi;
    p8_halves(w, lo, hi);
    const float2 a = xsv_unpack2<__half>(lo), b = xsv_unpack2<__half>(hi);
    s[0] += a.x; s[1] += a.y; s[2] += b.x; s[3] += b.y;
}

// Where 8 channels (from 8 piece on) of a token stand.
template <int D> __device__ __forceinline__ uint2* k_at(uint8_t* rec, int tok, int piece) {
    return reinterpret_cast<uint2*>(rec + Page8Rec<D>::K_CODES + (((tok >> 3) * (D / 64) + (piece >> 3)) * 32 + (tok & 7) * 4 + (piece >> 1 & 3)) * 16) + (piece & 1);
}
template <int D> __device__ __forceinline__ uint2* v_at(uint8_t* rec, int tok, int piece) {
    const int i = ((tok >> 4) * 4 + (tok >> 3 & 1) * 2 + (tok & 1)) * 32 + (tok >> 1 & 3);
    return reinterpret_cast<uint2*>(rec + Page8Rec<D>::V_CODES) + (D == 128 ? 2 * (i + 4 * (piece >> 1)) + (piece & 1) : i + 4 * piece);
}

// The mean key from a warp's sums of the page's key codes, channels (D / 32) lane on.
template <int D> __device__ __forceinline__ void store_mean(uint8_t* rec, const float (&s)[D / 32], float k_scale, int lane) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) top = fmaxf(top, fabsf(s[i]));
    top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)));
    const float inv = top > 0.f ? __fdiv_rn(127.f, top) : 0.f;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) w |= ((uint32_t)__float2int_rn(__fmul_rn(s[i], inv)) & 0xFFu) << (8 * i);
    if (D == 128) reinterpret_cast<uint32_t*>(rec + Page8Rec<D>::MEAN)[lane] = w;
    else reinterpret_cast<unsigned short*>(rec + Page8Rec<D>::MEAN)[lane] = (unsigned short)w;
    if (lane == 0) reinterpret_cast<float*>(rec + Page8Rec<D>::PARAMS)[2] = top * (k_scale * 0.015625f);
}

constexpr int WARPS = 4, THREADS = WARPS * 32;

constexpr int FEW = 16;                      // new tokens of a page up to which a warp stores them

// ---- a few new tokens of a page (decoding, the ends of prompts): a warp for one head of the page whose first new token is t
template <typename T, int D>
__device__ __forceinline__ void append_few(const Append8& p, const PagePlace& q, int t, int head) {
    using R = Page8Rec<D>;
    constexpr int PIECES = D / 8, ROWS = 32 / PIECES;         // rows of a turn
    const int lane = threadIdx.x & 31, run = min(XSV_PAGE - q.off, q.end - t), r_lane = lane / PIECES, piece = lane % PIECES;
    uint8_t* rec = page8_rec<D>(p.pool, q.page, head);
    const T* K = (const T*)p.K + (size_t)t * p.k_stride + (size_t)head * D + 8 * piece;
    const T* V = (const T*)p.V + (size_t)t * p.v_stride + (size_t)head * D + 8 * piece;
    float2* const params = reinterpret_cast<float2*>(rec + R::PARAMS);
    const float2 was = q.off > 0 ? *params : make_float2(0.f, 0.f);
    // the first turn's rows stay, further ones are read again
    uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
    if (r_lane < run) {
        k = load8(K + (size_t)r_lane * p.k_stride);
        v = load8(V + (size_t)r_lane * p.v_stride);
    }
    uint32_t mk = mag8(k, 0u), mv = mag8(v, 0u);
    for (int r = ROWS + r_lane; r < run; r += ROWS) {
        mk = mag8(load8(K + (size_t)r * p.k_stride), mk);
        mv = mag8(load8(V + (size_t)r * p.v_stride), mv);
    }
    mk = warp_mag(mk);
    mv = warp_mag(mv);
    int ek = exponent_of_mag<T>(mk), ev = exponent_of_mag<T>(mv);
    if (q.off > 0) {
        const int ok = p8_exponent_of(was.x), ov = p8_exponent_of(was.y);
        if (ek > ok) {                                         // a larger scale: what stands there moves to it
            for (int i = lane; i < (q.off + 7) / 8 * D; i += 32) {
                uint2* c = reinterpret_cast<uint2*>(rec + R::K_CODES) + i;
                *c = rescale8(*c, p8_pow2(max(ok - ek, -126)));
            }
        }
        if (ev > ov) {
            for (int i = lane; i < (q.off + 15) / 16 * 2 * D; i += 32) {
                uint2* c = reinterpret_cast<uint2*>(rec + R::V_CODES) + i;
                *c = rescale8(*c, p8_pow2(max(ov - ev, -126)));
            }
        }
        ek = max(ek, ok);
        ev = max(ev, ov);
        __syncwarp();                                          // (they touch places that new rows go to)
    }
    const Quant<T> qk(ek), qv(ev);
    for (int r = r_lane; r < run; r += ROWS) {
        if (r >= ROWS) {
            k = load8(K + (size_t)r * p.k_stride);
            v = load8(V + (size_t)r * p.v_stride);
        }
        if (max(mk, mv) > BOUND<T>) {
            k = bounded8<T>(k);
            v = bounded8<T>(v);
        }
        *k_at<D>(rec, q.off + r, piece) = codes8(k, qk);
        *v_at<D>(rec, q.off + r, piece) = codes8(v, qv);
    }
    if (lane == 0) *params = make_float2(p8_pow2(ek), p8_pow2(ev));
    if (q.off + run < XSV_PAGE) return;
    __syncwarp();
    float s[D / 32] = {};
#pragma unroll 16
    for (int tok = 0; tok < XSV_PAGE; ++tok) {
        if (D == 128) {
            add4(*(reinterpret_cast<const uint32_t*>(k_at<D>(rec, tok, lane >> 1)) + (lane & 1)), s);
        } else {
            uint32_t lo, hi;
            p8_halves(*(reinterpret_cast<const unsigned short*>(k_at<D>(rec, tok, lane >> 2)) + (lane & 3)), lo, hi);
            const float2 a = xsv_unpack2<__half>(lo);
            s[0] += a.x; s[1] += a.y;
        }
    }
    store_mean<D>(rec, s, p8_pow2(ek), lane);
}

// ---- more of them: a block looks for the first new tokens of pages among CHUNK ones and stores the keys, or the values, of p.across heads
// of each page, one after the other
constexpr int CHUNK = 32;

template <typename T, int D, bool KEYS>
__device__ __forceinline__ void append_pages(const Append8& p, int t_block, int head0, uint32_t (*s_mag)[WARPS], float (*s_sum)[D]) {
    using R = Page8Rec<D>;
    constexpr int PIECES = D / 8, ROWS = THREADS / PIECES, TURNS = XSV_PAGE / ROWS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, piece = tid % PIECES;
    // Row of a turn: a warp's rows are every other token, those that share sectors of the value codes.
    const int r0 = D == 128 ? 4 * (warp >> 1) + (warp & 1) + 2 * (lane >> 4) : 8 * (warp >> 1) + (warp & 1) + 2 * (lane >> 3);
    const int heads = min(p.across, p.pool.heads - head0);
    PagePlace mine{};
    const bool first = t_block + lane < p.n_tokens && place_of(p, t_block + lane, mine) && (t_block + lane == mine.begin || mine.off == 0) &&
                       min(XSV_PAGE - mine.off, mine.end - t_block - lane) > FEW;
    int buf = 0;
    for (uint32_t todo = __ballot_sync(0xFFFFFFFFu, first); todo; todo &= todo - 1) {      // the same for every warp
        const int from = __ffs(todo) - 1, t = t_block + from;
        const int off = __shfl_sync(0xFFFFFFFFu, mine.off, from), page = __shfl_sync(0xFFFFFFFFu, mine.page, from);
        const int run = min(XSV_PAGE - off, __shfl_sync(0xFFFFFFFFu, mine.end, from) - t);
        const bool full = off + run == XSV_PAGE;
        const long long stride = KEYS ? p.k_stride : p.v_stride;
        const T* x = (const T*)(KEYS ? p.K : p.V) + (long long)(t - off) * stride + (size_t)head0 * D + 8 * piece;
        uint8_t* rec = page8_rec<D>(p.pool, page, head0);
        // the heads, for a page that the call fills from its first row to its last (nothing else to ask about) and for others
        auto store = [&](auto whole_c) {
            constexpr bool WHOLE = decltype(whole_c)::value;
#pragma unroll 1
            for (int h = 0; h < heads; ++h, buf ^= 1, x += D, rec += R::BYTES) {
                float* const scale = reinterpret_cast<float*>(rec + R::PARAMS) + (KEYS ? 0 : 1);
                float was = 0.f;                               // of the tokens that stand in the page
                if (!WHOLE && off > 0) was = *scale;
                uint4 row[TURNS];
                uint32_t mag = 0u;
#pragma unroll
                for (int i = 0; i < TURNS; ++i) {
                    const int r = i * ROWS + r0;
                    if (!WHOLE) row[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (WHOLE || (r >= off && r < off + run)) row[i] = load8(x + (long long)r * stride);
                }
#pragma unroll
                for (int i = 0; i < TURNS; ++i) mag = mag8(row[i], mag);
                mag = warp_mag(mag);
                if (lane == 0) s_mag[buf][warp] = mag;
                __syncthreads();
                mag = max(max(s_mag[buf][0], s_mag[buf][1]), max(s_mag[buf][2], s_mag[buf][3]));
                if (mag > BOUND<T>)
#pragma unroll
                    for (int i = 0; i < TURNS; ++i) row[i] = bounded8<T>(row[i]);
                int e = exponent_of_mag<T>(mag);
                float f = 1.f;                                 // from the old scale to the new one
                if (!WHOLE && off > 0) {
                    const int o = p8_exponent_of(was);
                    f = p8_pow2(max(min(o - e, 0), -126));
                    e = max(e, o);
                }
                const Quant<T> q(e);
                float s[8] = {};
#pragma unroll
                for (int i = 0; i < TURNS; ++i) {
                    const int r = i * ROWS + r0;
                    if (!WHOLE && r >= off + run) continue;
                    uint2* const to = KEYS ? k_at<D>(rec, r, piece) : v_at<D>(rec, r, piece);
                    uint2 c;
                    if (WHOLE || r >= off) {
                        c = codes8(row[i], q);
                        *to = c;
                    } else {
                        c = make_uint2(0u, 0u);
                        if ((KEYS && full) || f != 1.f) c = *to;
                        if (f != 1.f) {
                            c = rescale8(c, f);
                            *to = c;
                        }
                    }
                    if (KEYS && (WHOLE || full)) { add4(c.x, s); add4(c.y, s + 4); }
                }
                if (tid == 0) *scale = p8_pow2(e);
                if (KEYS && (WHOLE || full)) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int o = 16; o >= PIECES; o >>= 1) s[i] += __shfl_xor_sync(0xFFFFFFFFu, s[i], o);
                    if (lane < PIECES) {
                        *reinterpret_cast<float4*>(&s_sum[warp][8 * piece]) = make_float4(s[0], s[1], s[2], s[3]);
                        *reinterpret_cast<float4*>(&s_sum[warp][8 * piece + 4]) = make_float4(s[4], s[5], s[6], s[7]);
                    }
                    __syncthreads();
                    if (warp == 0) {                           // (done before this warp passes the next barrier)
                        float m[D / 32];
#pragma unroll
                        for (int i = 0; i < D / 32; ++i) {
                            const int c = lane * (D / 32) + i;
                            m[i] = (s_sum[0][c] + s_sum[1][c]) + (s_sum[2][c] + s_sum[3][c]);
                        }
                        store_mean<D>(rec, m, p8_pow2(e), lane);
                    }
                }
            }
        };
        if (off == 0 && run == XSV_PAGE) store(std::true_type{});
        else store(std::false_type{});
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, D == 64 ? 9 : 7) page8_append_kernel(const __grid_constant__ Append8 p) {
    __shared__ uint32_t s_mag[2][WARPS];
    __shared__ __align__(16) float s_sum[WARPS][D];
    xsv_dep_release();
    xsv_dep_sync();
    if ((int)blockIdx.x < p.few_blocks) {
        // a sequence and WARPS heads: its first page here, and its last one
        const int parts = (p.pool.heads + WARPS - 1) / WARPS, seq = blockIdx.x / parts, head = (blockIdx.x - seq * parts) * WARPS + (threadIdx.x >> 5);
        const int begin = p.cu[seq], end = p.cu[seq + 1], total = p.total[seq];
        if (head >= p.pool.heads || begin < 0 || end <= begin || end > p.n_tokens || total < end - begin) return;
        const int last = (total - 1) / XSV_PAGE * XSV_PAGE - (total - (end - begin));        // the last page's first token, counted from `begin`
        for (int t = begin;; t = begin + last) {
            PagePlace q;
            if (place_of(p, t, q) && q.seq == seq && min(XSV_PAGE - q.off, q.end - t) <= FEW) append_few<T, D>(p, q, t, head);
            if (last <= 0 || t > begin) return;
        }
    }
    // the blocks for keys, which take longer, come first
    const int parts = (p.pool.heads + p.across - 1) / p.across, half = (gridDim.x - p.few_blocks) / 2, at = blockIdx.x - p.few_blocks, i = at < half ? at : at - half;
    const int t_block = i / parts * CHUNK, head0 = i % parts * p.across;
    if (at < half) append_pages<T, D, true>(p, t_block, head0, s_mag, s_sum);
    else append_pages<T, D, false>(p, t_block, head0, s_mag, s_sum);
}

// ------------------------------------------------------------------ reading back
struct Read8 {
    PoolView pool;
    const int* table;
    const int* total;
    const int* seq;
    const int* pos;
    void* K;
    void* V;
    int width, n_seqs, n_rows;
};

// Code pairs times the scale.  fp16 holds 65504 at most, the code of the largest inputs stands for 65536.
template <typename T> __device__ __forceinline__ uint32_t value2(uint32_t h, float s);
template <> __device__ __forceinline__ uint32_t value2<__half>(uint32_t h, float s) {
    const float2 f = xsv_unpack2<__half>(h);
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(f.y * s), "f"(f.x * s));
    return r;
}
template <> __device__ __forceinline__ uint32_t value2<__nv_bfloat16>(uint32_t h, float s) {
    const float2 f = xsv_unpack2<__half>(h);
    return xsv_pack2<__nv_bfloat16>(f.x * s, f.y * s);
}
template <typename T> __device__ __forceinline__ uint4 values8(uint32_t c0, uint32_t c1, float s) {
    uint32_t a, b, c, d;
    p8_halves(c0, a, b);
    p8_halves(c1, c, d);
    return make_uint4(value2<T>(a, s), value2<T>(b, s), value2<T>(c, s), value2<T>(d, s));
}

constexpr int READ_HEADS = 4;                 // heads of a token that a thread has on their way together

template <typename T, int D>
__global__ void __launch_bounds__(256) page8_read_kernel(const __grid_constant__ Read8 p) {
    using R = Page8Rec<D>;
    constexpr int PIECES = D / 8;
    xsv_dep_release();
    xsv_dep_sync();
    const int head0 = blockIdx.y * READ_HEADS, piece = threadIdx.x % PIECES;
    const long long r = (long long)blockIdx.x * (256 / PIECES) + threadIdx.x / PIECES;
    if (r >= p.n_rows) return;
    const int seq = p.seq[r], pos = p.pos[r];
    int page = -1;
    const int len = seq >= 0 && seq < p.n_seqs ? p.total[seq] : 0;
    if (pos >= 0 && pos < len && pos / XSV_PAGE < p.width) page = p.table[(size_t)seq * p.width + pos / XSV_PAGE];
    const bool is = page >= 0 && page < p.pool.n_pages;
    const int tok = pos & (XSV_PAGE - 1), heads = min(READ_HEADS, p.pool.heads - head0);
    float2 s[READ_HEADS];
    uint2 k[READ_HEADS], v[READ_HEADS];
#pragma unroll
    for (int h = 0; h < READ_HEADS; ++h) {
        s[h] = make_float2(0.f, 0.f);
        k[h] = v[h] = make_uint2(0u, 0u);
        if (is && h < heads) {
            uint8_t* rec = page8_rec<D>(p.pool, page, head0 + h);
            s[h] = *reinterpret_cast<const float2*>(rec + R::PARAMS);
            k[h] = *k_at<D>(rec, tok, piece);
            v[h] = *v_at<D>(rec, tok, piece);
        }
    }
#pragma unroll
    for (int h = 0; h < READ_HEADS; ++h) {
        if (h >= heads) break;
        const size_t to = ((size_t)r * p.pool.heads + head0 + h) * D + 8 * piece;
        *reinterpret_cast<uint4*>((T*)p.K + to) = values8<T>(k[h].x, k[h].y, s[h].x);
        *reinterpret_cast<uint4*>((T*)p.V + to) = values8<T>(v[h].x, v[h].y, s[h].y);
    }
}

}  // namespace

xsv_status xsv_page8_view(const xsv_page8_pool* pool, PoolView* v) {
    if (!pool || !pool->records) return XSV_ERR_ARG;
    if (pool->n_pages <= 0 || pool->kv_heads <= 0 || pool->kv_heads > 65535) return XSV_ERR_ARG;
    if (pool->head_dim != 64 && pool->head_dim != 128) return XSV_ERR_ARG;
    if (pool->dtype != XSV_F16 && pool->dtype != XSV_BF16) return XSV_ERR_ARG;
    if (pool->n_pages > XSV_PAGE_MAX_PAGES) return XSV_ERR_LIMIT;
    if ((uintptr_t)pool->records & 15) return XSV_ERR_SHAPE;
    *v = PoolView{(uint8_t*)pool->records, nullptr, pool->n_pages, XSV_PAGE_MAX_SEQS, pool->kv_heads};
    return XSV_OK;
}

extern "C" xsv_status xsv_page8_append(const xsv_page8_pool* pool, const void* K, const void* V, long long k_stride, long long v_stride, int n_tokens,
                                       const int* slot_map, const int* token_seq, const int* cu_new, const int* total_len, int n_seqs, void* stream) {
    Append8 p{};
    xsv_status s = xsv_page8_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_tokens < 0 || n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS) return XSV_ERR_ARG;
    if (n_tokens == 0) return XSV_OK;
    if (!K || !V || !slot_map || !token_seq || !cu_new || !total_len) return XSV_ERR_ARG;
    const long long row = (long long)pool->kv_heads * pool->head_dim;
    if (n_tokens > 1 && (k_stride < row || v_stride < row)) return XSV_ERR_ARG;
    if (((uintptr_t)K | (uintptr_t)V) & 15 || (k_stride | v_stride) & 7) return XSV_ERR_SHAPE;
    p.K = K; p.V = V; p.k_stride = k_stride; p.v_stride = v_stride;
    p.slot = slot_map; p.seq = token_seq; p.cu = cu_new; p.total = total_len;
    p.n_tokens = n_tokens; p.n_seqs = n_seqs;
    // A warp each for the pages that get at most 16 tokens, one or two a sequence, and blocks for the others, in one launch: a step may hold
    // decoding sequences and prompts.  8 heads of 128, all warps against all blocks: 128 sequences of 1 token 3.9 against 46 us, of 8 tokens 6.2
    // against 14, of 16 tokens 9.4 against 12.5; 4 sequences of 32 tokens, heads of 64: 5.9 against 4.2.  A block takes 4 heads (prompts of 19 735
    // tokens 14.5 us; 2 heads 15.7, 8 heads 20) while there are 8 blocks a multiprocessor.
    const long long chunks = ((long long)n_tokens + CHUNK - 1) / CHUNK, few = (long long)n_seqs * ((pool->kv_heads + WARPS - 1) / WARPS);
    p.across = 4;
    while (p.across > 1 && chunks * 2 * ((pool->kv_heads + p.across - 1) / p.across) < 8LL * xsv_sm_count()) p.across /= 2;
    const long long blocks = few + 2 * chunks * ((pool->kv_heads + p.across - 1) / p.across);
    if (blocks > 0x7FFFFFFFLL) return XSV_ERR_LIMIT;
    p.few_blocks = (int)few;
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, dim3((unsigned)blocks), dim3(THREADS), 0, (cudaStream_t)stream, p); };
    cudaError_t e;
    if (pool->dtype == XSV_F16) e = pool->head_dim == 64 ? go(page8_append_kernel<__half, 64>) : go(page8_append_kernel<__half, 128>);
    else e = pool->head_dim == 64 ? go(page8_append_kernel<__nv_bfloat16, 64>) : go(page8_append_kernel<__nv_bfloat16, 128>);
    if (e != cudaSuccess) return xsv_cuda_status(e);
    xsv_count_launch(1);
    return XSV_OK;
}

extern "C" xsv_status xsv_page8_read(const xsv_page8_pool* pool, const int* block_table, int table_width, const int* total_len, int n_seqs,
                                     const int* token_seq, const int* positions, int n_rows, void* K_out, void* V_out, void* stream) {
    Read8 p{};
    xsv_status s = xsv_page8_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_rows < 0 || n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS || table_width <= 0) return XSV_ERR_ARG;
    if (n_rows == 0) return XSV_OK;
    if (!block_table || !total_len || !token_seq || !positions || !K_out || !V_out) return XSV_ERR_ARG;
    if (((uintptr_t)K_out | (uintptr_t)V_out) & 15) return XSV_ERR_SHAPE;
    p.table = block_table; p.total = total_len; p.seq = token_seq; p.pos = positions; p.K = K_out; p.V = V_out;
    p.width = table_width; p.n_seqs = n_seqs; p.n_rows = n_rows;
    const int rows = 256 / (pool->head_dim / 8);
    const dim3 grid((unsigned)(((long long)n_rows + rows - 1) / rows), (pool->kv_heads + READ_HEADS - 1) / READ_HEADS);
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, grid, dim3(256), 0, (cudaStream_t)stream, p); };
    cudaError_t e;
    if (pool->dtype == XSV_F16) e = pool->head_dim == 64 ? go(page8_read_kernel<__half, 64>) : go(page8_read_kernel<__half, 128>);
    else e = pool->head_dim == 64 ? go(page8_read_kernel<__nv_bfloat16, 64>) : go(page8_read_kernel<__nv_bfloat16, 128>);
    if (e != cudaSuccess) return xsv_cuda_status(e);
    xsv_count_launch(1);
    return XSV_OK;
}
