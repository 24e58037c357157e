// Writing the 8-bit pages of the shared pool, and reading them back as values.
//
// xsv_page8_append: codes are written as their tokens come, without a 16-bit copy that waits for the page to fill: the block's
// scale is a power of two, so that a later token with a larger magnitude raises it and the codes that stand there are moved to
// the new scale (exact unless they become subnormal).  One block per (page, head) for prompts, one warp where most sequences
// bring a few tokens (decoding): the page's new rows are read once into registers, their largest magnitude is found, and they
// are stored as codes.  Whoever brings a page's last token also sums its key codes per channel, exactly (at most 64 * 448,
// in steps of 2^-9: 24 bits, so that no order of summation matters), for the mean key that a selection scores.
// Bound by HBM: 2 bytes read and 1 written per element.
//
// xsv_page8_read: a thread decodes 16 channels of one token.
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
};
__device__ __forceinline__ bool place_of(const Append8& p, int t, PagePlace& q) {
    return page_place(p.slot, p.seq, p.cu, p.total, p.n_tokens, p.n_seqs, p.pool.n_pages, t, q);
}

// Pairs of inputs brought to +-65504 (bf16: +-65536, whose code is the same); a NaN becomes the bound.
template <typename T> __device__ __forceinline__ uint32_t bounded2(uint32_t w);
template <> __device__ __forceinline__ uint32_t bounded2<__half>(uint32_t w) { return max2<__half>(min2<__half>(w, 0x7BFF7BFFu), 0xFBFFFBFFu); }
template <> __device__ __forceinline__ uint32_t bounded2<__nv_bfloat16>(uint32_t w) { return max2<__nv_bfloat16>(min2<__nv_bfloat16>(w, 0x47804780u), 0xC780C780u); }

// 16 channels of a row, and the larger of the magnitudes so far (as bit patterns, two a word: positive 16-bit floats compare
// like whole numbers).
struct Row16 { uint4 a, b; };
template <typename T> __device__ __forceinline__ Row16 load16(const void* x) {
    const uint4* p = reinterpret_cast<const uint4*>(x);
    Row16 r{p[0], p[1]};
    r.a = make_uint4(bounded2<T>(r.a.x), bounded2<T>(r.a.y), bounded2<T>(r.a.z), bounded2<T>(r.a.w));
    r.b = make_uint4(bounded2<T>(r.b.x), bounded2<T>(r.b.y), bounded2<T>(r.b.z), bounded2<T>(r.b.w));
    return r;
}
__device__ __forceinline__ uint32_t mag16(const Row16& r, uint32_t m) {
    constexpr uint32_t ABS = 0x7FFF7FFFu;
    m = __vmaxu2(m, __vmaxu2(__vmaxu2(r.a.x & ABS, r.a.y & ABS), __vmaxu2(r.a.z & ABS, r.a.w & ABS)));
    return __vmaxu2(m, __vmaxu2(__vmaxu2(r.b.x & ABS, r.b.y & ABS), __vmaxu2(r.b.z & ABS, r.b.w & ABS)));
}
template <typename T> __device__ __forceinline__ float mag_value(uint32_t m) { return xsv_unpack2<T>(max(m & 0xFFFFu, m >> 16)).x; }
template <typename T> __device__ __forceinline__ uint32_t codes4(uint32_t w0, uint32_t w1, float inv) {
    const float2 a = xsv_unpack2<T>(w0), b = xsv_unpack2<T>(w1);
    return p8_codes2(a.x * inv, a.y * inv) | p8_codes2(b.x * inv, b.y * inv) << 16;
}
template <typename T> __device__ __forceinline__ uint4 codes16(const Row16& r, float inv) {
    return make_uint4(codes4<T>(r.a.x, r.a.y, inv), codes4<T>(r.a.z, r.a.w, inv), codes4<T>(r.b.x, r.b.y, inv), codes4<T>(r.b.z, r.b.w, inv));
}
// four codes at another scale
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
    uint32_t lo, hi;
    p8_halves(w, lo, hi);
    const float2 a = xsv_unpack2<__half>(lo), b = xsv_unpack2<__half>(hi);
    return p8_codes2(a.x * f, a.y * f) | p8_codes2(b.x * f, b.y * f) << 16;
}
__device__ __forceinline__ uint4 rescale16(const uint4& w, float f) { return make_uint4(rescale4(w.x, f), rescale4(w.y, f), rescale4(w.z, f), rescale4(w.w, f)); }
__device__ __forceinline__ void add4(uint32_t w, float* s) {
    uint32_t lo, hi;
    p8_halves(w, lo, hi);
    const float2 a = xsv_unpack2<__half>(lo), b = xsv_unpack2<__half>(hi);
    s[0] += a.x; s[1] += a.y; s[2] += b.x; s[3] += b.y;
}

// Where 16 channels (from 16 piece on) of a token stand.
template <int D> __device__ __forceinline__ int k_at(int tok, int piece) { return (((tok >> 3) * (D / 64) + (piece >> 2)) * 32 + (tok & 7) * 4 + (piece & 3)) * 16; }
template <int D> __device__ __forceinline__ int v_index(int tok) { return ((tok >> 4) * 4 + (tok >> 3 & 1) * 2 + (tok & 1)) * 32 + (tok >> 1 & 3); }
template <int D> __device__ __forceinline__ uint4 v_load(const uint8_t* rec, int tok, int piece) {
    if (D == 128) return *reinterpret_cast<const uint4*>(rec + Page8Rec<D>::V_CODES + (v_index<D>(tok) + 4 * piece) * 16);
    const uint2 x = *reinterpret_cast<const uint2*>(rec + Page8Rec<D>::V_CODES + (v_index<D>(tok) + 8 * piece) * 8);
    const uint2 y = *reinterpret_cast<const uint2*>(rec + Page8Rec<D>::V_CODES + (v_index<D>(tok) + 8 * piece + 4) * 8);
    return make_uint4(x.x, x.y, y.x, y.y);
}
template <int D> __device__ __forceinline__ void v_store(uint8_t* rec, int tok, int piece, const uint4& c) {
    if (D == 128) {
        *reinterpret_cast<uint4*>(rec + Page8Rec<D>::V_CODES + (v_index<D>(tok) + 4 * piece) * 16) = c;
    } else {
        *reinterpret_cast<uint2*>(rec + Page8Rec<D>::V_CODES + (v_index<D>(tok) + 8 * piece) * 8) = make_uint2(c.x, c.y);
        *reinterpret_cast<uint2*>(rec + Page8Rec<D>::V_CODES + (v_index<D>(tok) + 8 * piece + 4) * 8) = make_uint2(c.z, c.w);
    }
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

// ---- a few tokens a sequence: a warp per (page, head), the page's first new token in the list
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) page8_append_few_kernel(const __grid_constant__ Append8 p) {
    using R = Page8Rec<D>;
    constexpr int PIECES = D / 16, ROWS = 32 / PIECES;        // rows of a turn
    xsv_dep_release();
    xsv_dep_sync();
    const int lane = threadIdx.x & 31, across = (p.pool.heads + WARPS - 1) / WARPS;
    const int t = blockIdx.x / across, head = (blockIdx.x - t * across) * WARPS + (threadIdx.x >> 5);
    PagePlace q;
    if (head >= p.pool.heads || !place_of(p, t, q) || !(t == q.begin || q.off == 0)) return;
    const int run = min(XSV_PAGE - q.off, q.end - t), r_lane = lane / PIECES, piece = lane % PIECES;
    uint8_t* rec = page8_rec<D>(p.pool, q.page, head);
    const T* K = (const T*)p.K + (size_t)t * p.k_stride + (size_t)head * D + 16 * piece;
    const T* V = (const T*)p.V + (size_t)t * p.v_stride + (size_t)head * D + 16 * piece;
    float2* const params = reinterpret_cast<float2*>(rec + R::PARAMS);
    const float2 was = q.off > 0 ? *params : make_float2(0.f, 0.f);
    // the first turn's rows stay, further ones are read again
    Row16 k{}, v{};
    if (r_lane < run) {
        k = load16<T>(K + (size_t)r_lane * p.k_stride);
        v = load16<T>(V + (size_t)r_lane * p.v_stride);
    }
    uint32_t mk = mag16(k, 0u), mv = mag16(v, 0u);
    for (int r = ROWS + r_lane; r < run; r += ROWS) {
        mk = mag16(load16<T>(K + (size_t)r * p.k_stride), mk);
        mv = mag16(load16<T>(V + (size_t)r * p.v_stride), mv);
    }
    mk = __reduce_max_sync(0xFFFFFFFFu, max(mk & 0xFFFFu, mk >> 16));
    mv = __reduce_max_sync(0xFFFFFFFFu, max(mv & 0xFFFFu, mv >> 16));
    int ek = p8_exponent(mag_value<T>(mk)), ev = p8_exponent(mag_value<T>(mv));
    if (q.off > 0) {
        const int ok = p8_exponent_of(was.x), ov = p8_exponent_of(was.y);
        if (ek > ok) {                                         // a larger scale: what stands there moves to it
            for (int i = lane; i < (q.off + 7) / 8 * (D / 64) * 32; i += 32) {
                uint4* c = reinterpret_cast<uint4*>(rec + R::K_CODES) + i;
                *c = rescale16(*c, p8_pow2(max(ok - ek, -126)));
            }
        }
        if (ev > ov) {
            for (int i = lane; i < (q.off + 15) / 16 * D; i += 32) {
                uint4* c = reinterpret_cast<uint4*>(rec + R::V_CODES) + i;
                *c = rescale16(*c, p8_pow2(max(ov - ev, -126)));
            }
        }
        ek = max(ek, ok);
        ev = max(ev, ov);
        __syncwarp();                                          // (they touch places that new rows go to)
    }
    const float ik = p8_pow2(-ek), iv = p8_pow2(-ev);
    for (int r = r_lane; r < run; r += ROWS) {
        if (r >= ROWS) {
            k = load16<T>(K + (size_t)r * p.k_stride);
            v = load16<T>(V + (size_t)r * p.v_stride);
        }
        *reinterpret_cast<uint4*>(rec + R::K_CODES + k_at<D>(q.off + r, piece)) = codes16<T>(k, ik);
        v_store<D>(rec, q.off + r, piece, codes16<T>(v, iv));
    }
    if (lane == 0) *params = make_float2(p8_pow2(ek), p8_pow2(ev));
    if (q.off + run < XSV_PAGE) return;
    __syncwarp();
    float s[D / 32] = {};
#pragma unroll 16
    for (int tok = 0; tok < XSV_PAGE; ++tok) {
        if (D == 128) {
            add4(*reinterpret_cast<const uint32_t*>(rec + k_at<D>(tok, lane >> 2) + 4 * (lane & 3)), s);
        } else {
            uint32_t lo, hi;
            p8_halves(*reinterpret_cast<const unsigned short*>(rec + k_at<D>(tok, lane >> 3) + 2 * (lane & 7)), lo, hi);
            const float2 a = xsv_unpack2<__half>(lo);
            s[0] += a.x; s[1] += a.y;
        }
    }
    store_mean<D>(rec, s, p8_pow2(ek), lane);
}

// ---- prompts: a block per (page, head), pages found among 32 new tokens
constexpr int CHUNK = 32;

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 4) page8_append_kernel(const __grid_constant__ Append8 p) {
    using R = Page8Rec<D>;
    constexpr int PIECES = D / 16, ROWS = THREADS / PIECES, TURNS = XSV_PAGE / ROWS;
    __shared__ uint32_t s_mag[2][2][WARPS];
    __shared__ __align__(16) float s_sum[WARPS][D];
    xsv_dep_release();
    xsv_dep_sync();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, piece = tid % PIECES, r0 = tid / PIECES;
    const int head = blockIdx.x % p.pool.heads, t_block = blockIdx.x / p.pool.heads * CHUNK;
    PagePlace mine{};
    const bool first = t_block + lane < p.n_tokens && place_of(p, t_block + lane, mine) && (t_block + lane == mine.begin || mine.off == 0);
    int buf = 0;
    for (uint32_t todo = __ballot_sync(0xFFFFFFFFu, first); todo; todo &= todo - 1, buf ^= 1) {      // the same for every warp
        const int from = __ffs(todo) - 1, t = t_block + from;
        const int off = __shfl_sync(0xFFFFFFFFu, mine.off, from), page = __shfl_sync(0xFFFFFFFFu, mine.page, from);
        const int run = min(XSV_PAGE - off, __shfl_sync(0xFFFFFFFFu, mine.end, from) - t);
        uint8_t* rec = page8_rec<D>(p.pool, page, head);
        const T* K = (const T*)p.K + (long long)(t - off) * p.k_stride + (size_t)head * D + 16 * piece;
        const T* V = (const T*)p.V + (long long)(t - off) * p.v_stride + (size_t)head * D + 16 * piece;
        float2* const params = reinterpret_cast<float2*>(rec + R::PARAMS);
        const float2 was = off > 0 ? *params : make_float2(0.f, 0.f);
        Row16 k[TURNS] = {}, v[TURNS] = {};
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int r = i * ROWS + r0;
            if (r >= off && r < off + run) {
                k[i] = load16<T>(K + (long long)r * p.k_stride);
                v[i] = load16<T>(V + (long long)r * p.v_stride);
            }
        }
        uint32_t mk = 0u, mv = 0u;
#pragma unroll
        for (int i = 0; i < TURNS; ++i) { mk = mag16(k[i], mk); mv = mag16(v[i], mv); }
        mk = __reduce_max_sync(0xFFFFFFFFu, max(mk & 0xFFFFu, mk >> 16));
        mv = __reduce_max_sync(0xFFFFFFFFu, max(mv & 0xFFFFu, mv >> 16));
        if (lane == 0) { s_mag[buf][0][warp] = mk; s_mag[buf][1][warp] = mv; }
        __syncthreads();
        mk = max(max(s_mag[buf][0][0], s_mag[buf][0][1]), max(s_mag[buf][0][2], s_mag[buf][0][3]));
        mv = max(max(s_mag[buf][1][0], s_mag[buf][1][1]), max(s_mag[buf][1][2], s_mag[buf][1][3]));
        int ek = p8_exponent(mag_value<T>(mk)), ev = p8_exponent(mag_value<T>(mv));
        float fk = 1.f, fv = 1.f;                              // from the old scale to the new one
        if (off > 0) {
            const int ok = p8_exponent_of(was.x), ov = p8_exponent_of(was.y);
            fk = p8_pow2(max(min(ok - ek, 0), -126));
            fv = p8_pow2(max(min(ov - ev, 0), -126));
            ek = max(ek, ok);
            ev = max(ev, ov);
        }
        const float ik = p8_pow2(-ek), iv = p8_pow2(-ev);
        const bool full = off + run == XSV_PAGE;
        float s[16] = {};
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int r = i * ROWS + r0;
            if (r >= off + run) continue;
            uint8_t* const k_to = rec + R::K_CODES + k_at<D>(r, piece);
            uint4 c;
            if (r >= off) {
                c = codes16<T>(k[i], ik);
                *reinterpret_cast<uint4*>(k_to) = c;
                v_store<D>(rec, r, piece, codes16<T>(v[i], iv));
            } else {
                c = make_uint4(0u, 0u, 0u, 0u);
                if (full || fk != 1.f) c = *reinterpret_cast<const uint4*>(k_to);
                if (fk != 1.f) {
                    c = rescale16(c, fk);
                    *reinterpret_cast<uint4*>(k_to) = c;
                }
                if (fv != 1.f) v_store<D>(rec, r, piece, rescale16(v_load<D>(rec, r, piece), fv));
            }
            if (full) { add4(c.x, s); add4(c.y, s + 4); add4(c.z, s + 8); add4(c.w, s + 12); }
        }
        if (tid == 0) *params = make_float2(p8_pow2(ek), p8_pow2(ev));
        if (full) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int o = PIECES; o < 32; o <<= 1) s[i] += __shfl_xor_sync(0xFFFFFFFFu, s[i], o);
            if (lane < PIECES)
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(&s_sum[warp][16 * piece + 4 * i]) = make_float4(s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]);
            __syncthreads();
            if (warp == 0) {                                   // (done before this warp passes the next page's barrier)
                float m[D / 32];
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const int c = lane * (D / 32) + i;
                    m[i] = (s_sum[0][c] + s_sum[1][c]) + (s_sum[2][c] + s_sum[3][c]);
                }
                store_mean<D>(rec, m, p8_pow2(ek), lane);
            }
        }
    }
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

template <typename T, int D>
__global__ void __launch_bounds__(256) page8_read_kernel(const __grid_constant__ Read8 p) {
    using R = Page8Rec<D>;
    constexpr int PIECES = D / 16;
    xsv_dep_release();
    xsv_dep_sync();
    const int head = blockIdx.y, piece = threadIdx.x % PIECES;
    const long long r = (long long)blockIdx.x * (256 / PIECES) + threadIdx.x / PIECES;
    if (r >= p.n_rows) return;
    const int seq = p.seq[r], pos = p.pos[r];
    int page = -1;
    const int len = seq >= 0 && seq < p.n_seqs ? p.total[seq] : 0;
    if (pos >= 0 && pos < len && pos / XSV_PAGE < p.width) page = p.table[(size_t)seq * p.width + pos / XSV_PAGE];
    uint4 out[4] = {};
    if (page >= 0 && page < p.pool.n_pages) {
        const uint8_t* rec = page8_rec<D>(p.pool, page, head);
        const int tok = pos % XSV_PAGE;
        const float2 s = *reinterpret_cast<const float2*>(rec + R::PARAMS);
        const uint4 k = *reinterpret_cast<const uint4*>(rec + R::K_CODES + k_at<D>(tok, piece)), v = v_load<D>(rec, tok, piece);
        out[0] = values8<T>(k.x, k.y, s.x); out[1] = values8<T>(k.z, k.w, s.x);
        out[2] = values8<T>(v.x, v.y, s.y); out[3] = values8<T>(v.z, v.w, s.y);
    }
    const size_t to = ((size_t)r * p.pool.heads + head) * D + 16 * piece;
    uint4* const k_to = reinterpret_cast<uint4*>((T*)p.K + to);
    uint4* const v_to = reinterpret_cast<uint4*>((T*)p.V + to);
    k_to[0] = out[0]; k_to[1] = out[1];
    v_to[0] = out[2]; v_to[1] = out[3];
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
    const bool few = (long long)n_tokens <= 4LL * n_seqs;
    const long long blocks = few ? (long long)n_tokens * ((pool->kv_heads + WARPS - 1) / WARPS) : ((long long)n_tokens + CHUNK - 1) / CHUNK * pool->kv_heads;
    if (blocks > 0x7FFFFFFFLL) return XSV_ERR_LIMIT;
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, dim3((unsigned)blocks), dim3(THREADS), 0, (cudaStream_t)stream, p); };
    cudaError_t e;
    if (pool->dtype == XSV_F16) {
        if (few) e = pool->head_dim == 64 ? go(page8_append_few_kernel<__half, 64>) : go(page8_append_few_kernel<__half, 128>);
        else e = pool->head_dim == 64 ? go(page8_append_kernel<__half, 64>) : go(page8_append_kernel<__half, 128>);
    } else {
        if (few) e = pool->head_dim == 64 ? go(page8_append_few_kernel<__nv_bfloat16, 64>) : go(page8_append_few_kernel<__nv_bfloat16, 128>);
        else e = pool->head_dim == 64 ? go(page8_append_kernel<__nv_bfloat16, 64>) : go(page8_append_kernel<__nv_bfloat16, 128>);
    }
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
    const int rows = 256 / (pool->head_dim / 16);
    const dim3 grid((unsigned)(((long long)n_rows + rows - 1) / rows), pool->kv_heads);
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, grid, dim3(256), 0, (cudaStream_t)stream, p); };
    cudaError_t e;
    if (pool->dtype == XSV_F16) e = pool->head_dim == 64 ? go(page8_read_kernel<__half, 64>) : go(page8_read_kernel<__half, 128>);
    else e = pool->head_dim == 64 ? go(page8_read_kernel<__nv_bfloat16, 64>) : go(page8_read_kernel<__nv_bfloat16, 128>);
    if (e != cudaSuccess) return xsv_cuda_status(e);
    xsv_count_launch(1);
    return XSV_OK;
}
