// Writing the pages of the shared pool, and reading them back as values.
//
// xsv_page_append: one block per (new tokens of one page, head), or, where a few tokens do not fill their page
// (decoding), one warp.  Values are quantised per token over 64 channels as they come and merged into the page's code
// words (a token is one byte of each word it touches); keys need all 64 tokens of a page for their per-channel scale,
// so a page's keys wait in the sequence's tail, in 16 bits, and are quantised by the call that brings the page's last
// token.  The tail has two halves, by the page's parity: the page
// that is completed is read from one while the page after it starts in the other.  Bound by HBM for prompts (2 bytes
// read, 72/128 written per element); the thread layout makes both packings local to a thread -- a thread's 8 rows x
// 8 channels of keys (rows 8 i + g) are whole code words, and so are 4 tokens x 8 channels of values -- so codes never
// pass through shared memory, only the column minima and maxima do.
//
// xsv_page_read: one block per (32 listed tokens, head); a thread decodes 8 channels of one token, so that a page's
// record is fetched once into L1 for the rows that share its sectors and the outputs are written 16 bytes a thread.
//
// Measured.  Append of 19 735 prompt tokens, 8 heads of 64, fp16: 26 us, 2.0 TB/s (first version 140); of one token for each of 256
// sequences, 8 heads of 128, bf16: 8.6 us, of which a page that is filled takes 5 (38).  Bound by latency: a block goes
// through lookup, values, keys and two barriers one after the other, and registers allow 20 warps a multiprocessor;
// fetching the keys ahead of the values spilled (29 us), packed float32 arithmetic changed nothing.  Reading the same tokens
// back: 14 us, 3.7 TB/s, and 8150 tokens of 8 heads of 128: 11.7 us, 4.5 TB/s.
#include "../../include/xsv.h"
#include "page_layout.cuh"
#include "xsv_kernels.h"

namespace {

struct Append {
    PoolView pool;
    const void* K;
    const void* V;
    long long k_stride, v_stride;
    const int* slot;
    const int* seq;
    const int* cu;
    const int* total;
    int n_tokens, n_seqs, chunk, few_blocks, few_heads;     // few_: blocks of one token, groups of heads that they are split into
};

template <typename T> __device__ __forceinline__ void unpack8(const uint4& w, float (&o)[8]) {
    const float2 a = xsv_unpack2<T>(w.x), b = xsv_unpack2<T>(w.y), c = xsv_unpack2<T>(w.z), d = xsv_unpack2<T>(w.w);
    o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y; o[4] = c.x; o[5] = c.y; o[6] = d.x; o[7] = d.y;
}

// Where new token t lands.  False for a token without a place, or with one that contradicts the lengths.
struct Place { int seq, begin, end, page, off, pos; };
__device__ __forceinline__ bool place_of(const Append& p, int t, Place& q) {
    const int slot = p.slot[t];
    q.seq = p.seq[t];
    if (slot < 0 || q.seq < 0 || q.seq >= p.n_seqs || q.seq >= p.pool.max_seqs) return false;
    q.begin = p.cu[q.seq];
    q.end = p.cu[q.seq + 1];
    q.page = slot / XSV_PAGE;
    q.off = slot % XSV_PAGE;
    if (q.begin < 0 || q.begin > t || q.end <= t || q.end > p.n_tokens || q.page >= p.pool.n_pages) return false;
    q.pos = p.total[q.seq] - (q.end - t);
    return q.pos >= q.off && q.pos - (t - q.begin) >= 0 && q.pos % XSV_PAGE == q.off;
}

// What codes are computed from: bf16 values beyond fp16 are brought to +-65504, fp16 ones have no such values.
template <typename T> __device__ __forceinline__ float code_input(float x);
template <> __device__ __forceinline__ float code_input<__half>(float x) { return x; }
template <> __device__ __forceinline__ float code_input<__nv_bfloat16>(float x) { return clamp_half(x); }
template <typename T> __device__ __forceinline__ void codes8(const float (&x)[8], float s, float inv, float z, uint32_t (&c)[8]) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = code_input<T>(x[i]);
    page_codes(y, s, inv, z, c);
}
template <typename T> __device__ __forceinline__ void range8(const uint4& v, float& mn, float& mx) {
    const float2 lo = xsv_unpack2<T>(min2<T>(min2<T>(v.x, v.y), min2<T>(v.z, v.w)));
    const float2 hi = xsv_unpack2<T>(max2<T>(max2<T>(v.x, v.y), max2<T>(v.z, v.w)));
    mn = fminf(lo.x, lo.y);
    mx = fmaxf(hi.x, hi.y);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {                       // the 8 pieces of 64 channels are 8 neighbouring lanes
        mn = fminf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, o));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
    }
}

constexpr int FEW = 8;                       // new tokens of a page up to which one warp appends them

template <typename T, int D>
__global__ void __launch_bounds__(D, D == 128 ? 5 : 10) page_append_kernel(const __grid_constant__ Append p) {
    using R = PageRec<D>;
    constexpr int C = D / 8, W = D / 32;     // 8-channel pieces of a row, warps
    __shared__ uint32_t s_mn[8][D / 2], s_mx[8][D / 2];
    __shared__ float s_scale[D], s_zero[D], s_inv[D];
    xsv_dep_release();
    xsv_dep_sync();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // the chunk's tokens that are the first new ones of their page; every warp finds the same
    Place mine{};
    bool first = false, few = false;
    // The first blocks (decoding) have a token and a head a warp and take the few-token pages, the others `chunk` tokens and a head.
    const bool one = (int)blockIdx.x < p.few_blocks;
    const int index = one ? blockIdx.x : blockIdx.x - p.few_blocks, across = one ? p.few_heads : p.pool.heads;
    const int t_block = index / across * (one ? 1 : p.chunk), head0 = index % across * (one ? W : 1), head1 = min(p.pool.heads, head0 + (one ? W : 1));
    const int t_lane = t_block + lane;
    if (lane < (one ? 1 : p.chunk) && t_lane < p.n_tokens) first = place_of(p, t_lane, mine) && (t_lane == mine.begin || mine.off == 0);
    if (first) {
        const int run = min(XSV_PAGE - mine.off, mine.end - t_lane);
        few = run <= FEW && mine.off + run < XSV_PAGE;
    }
    const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, first), fews = __ballot_sync(0xFFFFFFFFu, few);
    auto place_at = [&](int from) {
        Place q;
        q.seq = __shfl_sync(0xFFFFFFFFu, mine.seq, from);
        q.begin = __shfl_sync(0xFFFFFFFFu, mine.begin, from);
        q.end = __shfl_sync(0xFFFFFFFFu, mine.end, from);
        q.page = __shfl_sync(0xFFFFFFFFu, mine.page, from);
        q.off = __shfl_sync(0xFFFFFFFFu, mine.off, from);
        q.pos = __shfl_sync(0xFFFFFFFFu, mine.pos, from);
        return q;
    };
    // The last, unfilled page's keys go to the tail half of its parity.  Where the sequence's first page here still
    // reads old keys from that half, the block of that first page writes them, after its reads.
    auto handed_on = [&](const Place& q, int t) {
        const int p0 = q.pos - (t - q.begin), first_no = p0 / XSV_PAGE, last_no = (q.pos + q.end - t) / XSV_PAGE;
        return p0 % XSV_PAGE != 0 && last_no > first_no && ((last_no - first_no) & 1) == 0;
    };

    // ---- a few tokens that do not fill their page (decoding): a warp each, every lane 8 channels of a token
    int turn = 0;
    for (uint32_t todo = one || p.few_blocks == 0 ? fews : 0; todo; todo &= todo - 1) {
        const int from = __ffs(todo) - 1, t = t_block + from;
        const Place q = place_at(from);
        for (int head = head0; head < head1; ++head, ++turn) {
            if (turn % W != warp) continue;
            const int run = min(XSV_PAGE - q.off, q.end - t), page_no = q.pos / XSV_PAGE, piece = lane % C;
            const bool skip_keys = handed_on(q, t) && page_no != (q.pos - (t - q.begin)) / XSV_PAGE;
            uint8_t* rec = page_rec<D>(p.pool, q.page, head);
            T* tail = tail_rows<T, D>(p.pool, q.seq, page_no, head) + 8 * piece;
            for (int r0 = 0; r0 < run; r0 += 32 / C) {          // the same for the whole warp
                const int r = r0 + lane / C, tok = q.off + r;
                const bool live = r < run;
                uint4 k = make_uint4(0, 0, 0, 0), v = k;
                if (live) {
                    k = *reinterpret_cast<const uint4*>((const T*)p.K + (size_t)(t + r) * p.k_stride + (size_t)head * D + 8 * piece);
                    v = *reinterpret_cast<const uint4*>((const T*)p.V + (size_t)(t + r) * p.v_stride + (size_t)head * D + 8 * piece);
                }
                if (live && !skip_keys) *reinterpret_cast<uint4*>(tail + (size_t)tok * D) = k;
                float mn, mx, x[8];
                range8<T>(v, mn, mx);
                __half hs, hz;
                page_params(clamp_half(mn), clamp_half(mx), hs, hz);
                const float s = __half2float(hs), z = __half2float(hz);
                uint32_t c[8];
                unpack8<T>(v, x);
                codes8<T>(x, s, page_inverse(s), z, c);
                if (live) {
                    // the token's byte of four words: [k = tok / 16][c][g][j = tok % 8 / 2][m], byte 2 (tok % 2) + tok / 8 % 2
                    uint8_t* at = rec + R::V_CODES + (((tok / 16) * (D / 64) + piece / 8) * 32 + (piece % 8) * 4 + tok % 8 / 2) * 16 + 2 * (tok % 2) + tok / 8 % 2;
#pragma unroll
                    for (int m = 0; m < 4; ++m) at[4 * m] = (uint8_t)(c[2 * m] | c[2 * m + 1] << 4);
                    if (piece % 8 == 0) {
                        const int i = (piece / 8) * 64 + (tok % 8) * 8 + tok / 8;
                        reinterpret_cast<__half*>(rec + R::V_SCALE)[i] = hs;
                        reinterpret_cast<__half*>(rec + R::V_ZERO)[i] = hz;
                    }
                }
            }
        }
    }

    // ---- the others: the whole block, one page and head at a time
    const int piece = tid % C, g = tid / C;
    for (uint32_t todo = one ? 0 : firsts & ~fews; todo; todo &= todo - 1) {
        const int from = __ffs(todo) - 1, t = t_block + from;
        const Place q = place_at(from);
        const int run = min(XSV_PAGE - q.off, q.end - t), total = q.pos + q.end - t, page_no = q.pos / XSV_PAGE;
        const bool full = q.off + run == XSV_PAGE, handed = handed_on(q, t);
        const int first_no = (q.pos - (t - q.begin)) / XSV_PAGE, last_no = total / XSV_PAGE;
#pragma unroll 1
        for (int head = head0; head < head1; ++head) {
            uint8_t* rec = page_rec<D>(p.pool, q.page, head);
            const T* K = (const T*)p.K + (size_t)head * D + 8 * piece;
            const T* V = (const T*)p.V + (size_t)head * D + 8 * piece;
            // values: 4 tokens x 8 channels a thread, twice
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const int combo = g + 8 * half, tok0 = 16 * (combo >> 2) + 2 * (combo & 3);
                uint4 raw[4];
                uint32_t mask = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int tok = tok0 + 8 * (b & 1) + (b >> 1);
                    raw[b] = make_uint4(0, 0, 0, 0);
                    if (tok >= q.off && tok < q.off + run) {
                        raw[b] = *reinterpret_cast<const uint4*>(V + (size_t)(t + tok - q.off) * p.v_stride);
                        mask |= 0xFFu << (8 * b);
                    }
                }
                if (!__any_sync(0xFFFFFFFFu, mask != 0)) continue;
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll 2
                for (int b = 0; b < 4; ++b) {
                    if (!__any_sync(0xFFFFFFFFu, mask >> (8 * b) & 1u)) continue;
                    const uint4 v = b == 0 ? raw[0] : b == 1 ? raw[1] : b == 2 ? raw[2] : raw[3];
                    float mn, mx, x[8];
                    range8<T>(v, mn, mx);
                    __half hs, hz;
                    page_params(clamp_half(mn), clamp_half(mx), hs, hz);
                    const float s = __half2float(hs), z = __half2float(hz);
                    uint32_t c[8];
                    unpack8<T>(v, x);
                    codes8<T>(x, s, page_inverse(s), z, c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] += (c[2 * i] + (c[2 * i + 1] << 4)) << (8 * b);
                    if (piece % 8 == 0 && (mask >> (8 * b) & 1u)) {
                        const int tok = tok0 + 8 * (b & 1) + (b >> 1), at = (piece / 8) * 64 + (tok % 8) * 8 + tok / 8;
                        reinterpret_cast<__half*>(rec + R::V_SCALE)[at] = hs;
                        reinterpret_cast<__half*>(rec + R::V_ZERO)[at] = hz;
                    }
                }
                if (mask) {
                    uint4* at = reinterpret_cast<uint4*>(rec + R::V_CODES + (((combo >> 2) * (D / 64) + piece / 8) * 32 + (piece % 8) * 4 + (combo & 3)) * 16);
                    uint4 old = make_uint4(0, 0, 0, 0);
                    if (mask != 0xFFFFFFFFu) old = *at;
                    *at = make_uint4((w[0] & mask) | (old.x & ~mask), (w[1] & mask) | (old.y & ~mask), (w[2] & mask) | (old.z & ~mask),
                                     (w[3] & mask) | (old.w & ~mask));
                }
            }
            // keys
            if (!full) {
                if (!(handed && page_no != first_no)) {
                    T* tail = tail_rows<T, D>(p.pool, q.seq, page_no, head) + 8 * piece;
                    for (int r = g; r < run; r += 8)
                        *reinterpret_cast<uint4*>(tail + (size_t)(q.off + r) * D) = *reinterpret_cast<const uint4*>(K + (size_t)(t + r) * p.k_stride);
                }
                continue;
            }
            uint4 row[8];
            {
                const T* tail = tail_rows<T, D>(p.pool, q.seq, page_no, head) + 8 * piece;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 8 * i + g;
                    row[i] = *reinterpret_cast<const uint4*>(r < q.off ? tail + (size_t)r * D : K + (size_t)(t + r - q.off) * p.k_stride);
                }
            }
            {
                uint4 mn = row[0], mx = row[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) {
                    mn = make_uint4(min2<T>(mn.x, row[i].x), min2<T>(mn.y, row[i].y), min2<T>(mn.z, row[i].z), min2<T>(mn.w, row[i].w));
                    mx = make_uint4(max2<T>(mx.x, row[i].x), max2<T>(mx.y, row[i].y), max2<T>(mx.z, row[i].z), max2<T>(mx.w, row[i].w));
                }
                *reinterpret_cast<uint4*>(&s_mn[g][4 * piece]) = mn;
                *reinterpret_cast<uint4*>(&s_mx[g][4 * piece]) = mx;
            }
            __syncthreads();
            if (tid < D / 2) {
                uint32_t mn = s_mn[0][tid], mx = s_mx[0][tid];
#pragma unroll
                for (int i = 1; i < 8; ++i) { mn = min2<T>(mn, s_mn[i][tid]); mx = max2<T>(mx, s_mx[i][tid]); }
                const float2 lo = xsv_unpack2<T>(mn), hi = xsv_unpack2<T>(mx);
                __half s0, z0, s1, z1;
                page_params(clamp_half(lo.x), clamp_half(hi.x), s0, z0);
                page_params(clamp_half(lo.y), clamp_half(hi.y), s1, z1);
                reinterpret_cast<__half2*>(rec + R::K_SCALE)[tid] = __halves2half2(s0, s1);
                reinterpret_cast<__half2*>(rec + R::K_ZERO)[tid] = __halves2half2(z0, z1);
                const float f0 = __half2float(s0), f1 = __half2float(s1);
                reinterpret_cast<float2*>(s_scale)[tid] = make_float2(f0, f1);
                reinterpret_cast<float2*>(s_zero)[tid] = make_float2(__half2float(z0), __half2float(z1));
                reinterpret_cast<float2*>(s_inv)[tid] = make_float2(page_inverse(f0), page_inverse(f1));
            }
            __syncthreads();
            // channel c of the piece: step 2 (piece / 4) + c / 4, byte 2 (c % 2) + (c % 4) / 2; row 8 i + g: word i / 2,
            // nibble i % 2.  Two channels a turn, the rows' next pair moved up after it: unrolled, this is more code than the
            // instruction cache holds.
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll 1
            for (int c = 0; c < 8; c += 2) {
                const float2 s = *reinterpret_cast<const float2*>(&s_scale[8 * piece + c]), z = *reinterpret_cast<const float2*>(&s_zero[8 * piece + c]),
                             inv = *reinterpret_cast<const float2*>(&s_inv[8 * piece + c]);
                float x0[8], x1[8];
                uint32_t c0[8], c1[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 two = xsv_unpack2<T>(row[i].x);
                    x0[i] = two.x;
                    x1[i] = two.y;
                    row[i].x = row[i].y; row[i].y = row[i].z; row[i].z = row[i].w;
                }
                codes8<T>(x0, s.x, inv.x, z.x, c0);
                codes8<T>(x1, s.y, inv.y, z.y, c1);
                const int sh = 4 * (c & 2);                     // byte (c % 4) / 2, and two bytes up for the second channel
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] += (c0[2 * i] + (c0[2 * i + 1] << 4) + (c1[2 * i] << 16) + (c1[2 * i + 1] << 20)) << sh;
                if (c & 2) {
                    *reinterpret_cast<uint4*>(rec + R::K_CODES + ((2 * (piece / 4) + c / 4) * 32 + g * 4 + piece % 4) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                    w[0] = w[1] = w[2] = w[3] = 0;
                }
            }
            if (handed && page_no == first_no) {                // after the barriers: the old keys have been read
                const int left = total % XSV_PAGE;
                T* tail = tail_rows<T, D>(p.pool, q.seq, last_no, head) + 8 * piece;
                for (int r = g; r < left; r += 8)
                    *reinterpret_cast<uint4*>(tail + (size_t)r * D) = *reinterpret_cast<const uint4*>(K + (size_t)(q.end - left + r) * p.k_stride);
            }
        }
    }
}

struct Read {
    PoolView pool;
    const int* table;
    const int* total;
    const int* seq;
    const int* pos;
    void* K;
    void* V;
    int width, n_seqs, n_rows;
};

constexpr int READ_ROWS = 32;                // rows of a block
constexpr uint32_t LOW = 0x000F000Fu;
// Two codes (in the halves of a word) times scale plus offset, rounded once: fp16 by one fused operation, bf16 from float32.
// 1024 + code, as fp16 bits, minus 1024 is the code exactly.
template <typename T> __device__ __forceinline__ uint32_t value2(uint32_t codes, uint32_t s, uint32_t z);
template <> __device__ __forceinline__ uint32_t value2<__half>(uint32_t codes, uint32_t s, uint32_t z) {
    uint32_t c = codes | 0x64006400u, d;
    asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(c) : "r"(0x64006400u));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(c), "r"(s), "r"(z));
    return d;
}
template <> __device__ __forceinline__ uint32_t value2<__nv_bfloat16>(uint32_t codes, uint32_t s, uint32_t z) {
    const float2 fs = xsv_unpack2<__half>(s), fz = xsv_unpack2<__half>(z);
    const float c0 = __fadd_rn(__uint_as_float(codes & 15u | 0x4B000000u), -8388608.f), c1 = __fadd_rn(__uint_as_float(codes >> 16 | 0x4B000000u), -8388608.f);
    return xsv_pack2<__nv_bfloat16>(fmaf(c0, fs.x, fz.x), fmaf(c1, fs.y, fz.y));
}

template <typename T, int D>
__global__ void __launch_bounds__(256) page_read_kernel(const __grid_constant__ Read p) {
    using R = PageRec<D>;
    constexpr int C = D / 8;
    xsv_dep_release();
    xsv_dep_sync();
    const int head = blockIdx.y, piece = threadIdx.x % C;
    const int r1 = min(p.n_rows, (int)(blockIdx.x + 1) * READ_ROWS);
#pragma unroll
    for (int i = 0; i < READ_ROWS * C / 256; ++i) {
        const int r = blockIdx.x * READ_ROWS + i * (256 / C) + threadIdx.x / C;
        if (r >= r1) break;
        const int seq = p.seq[r], pos = p.pos[r];
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        int page = -1;
        const int len = seq >= 0 && seq < p.n_seqs && seq < p.pool.max_seqs ? p.total[seq] : 0;
        if (pos >= 0 && pos < len && pos / XSV_PAGE < p.width) page = p.table[(size_t)seq * p.width + pos / XSV_PAGE];
        if (page >= 0 && page < p.pool.n_pages) {
            const uint8_t* rec = page_rec<D>(p.pool, page, head);
            const int tok = pos % XSV_PAGE, g = tok % 8;
            if (pos / XSV_PAGE == len / XSV_PAGE) {              // the unfilled page: keys as they came
                k = *reinterpret_cast<const uint4*>(tail_rows<T, D>(p.pool, seq, pos / XSV_PAGE, head) + (size_t)tok * D + 8 * piece);
            } else {
                const uint4 s = *reinterpret_cast<const uint4*>(rec + R::K_SCALE + 16 * piece);
                const uint4 z = *reinterpret_cast<const uint4*>(rec + R::K_ZERO + 16 * piece);
                const uint8_t* at = rec + R::K_CODES + (2 * (piece / 4) * 32 + g * 4 + piece % 4) * 16 + (tok / 16) * 4;
                const int sh = tok / 8 % 2 * 4;
                const uint32_t w0 = *reinterpret_cast<const uint32_t*>(at) >> sh, w1 = *reinterpret_cast<const uint32_t*>(at + 512) >> sh;
                k = make_uint4(value2<T>(w0 & LOW, s.x, z.x), value2<T>(w0 >> 8 & LOW, s.y, z.y), value2<T>(w1 & LOW, s.z, z.z), value2<T>(w1 >> 8 & LOW, s.w, z.w));
            }
            const int at = (piece / 8) * 64 + g * 8 + tok / 8;
            uint32_t s = reinterpret_cast<const unsigned short*>(rec + R::V_SCALE)[at], z = reinterpret_cast<const unsigned short*>(rec + R::V_ZERO)[at];
            s |= s << 16;
            z |= z << 16;
            const uint4 w = *reinterpret_cast<const uint4*>(rec + R::V_CODES + (((tok / 16) * (D / 64) + piece / 8) * 32 + (piece % 8) * 4 + tok % 8 / 2) * 16);
            // the token's byte at both ends of a word: its low nibble below, its high nibble four bits up above
            const uint32_t sel = 0x4040u + 0x0101u * (uint32_t)(2 * (tok % 2) + tok / 8 % 2);
            auto pair = [&](uint32_t word) {
                const uint32_t x = __byte_perm(word, 0, sel);
                return (x & 0xFu) | (x >> 4 & 0xF0000u);
            };
            v = make_uint4(value2<T>(pair(w.x), s, z), value2<T>(pair(w.y), s, z), value2<T>(pair(w.z), s, z), value2<T>(pair(w.w), s, z));
        }
        const size_t to = ((size_t)r * p.pool.heads + head) * D + 8 * piece;
        *reinterpret_cast<uint4*>((T*)p.K + to) = k;
        *reinterpret_cast<uint4*>((T*)p.V + to) = v;
    }
}

}  // namespace


xsv_status xsv_pool_view(const xsv_page_pool* pool, PoolView* v) {
    if (!pool || !pool->records || !pool->k_tail) return XSV_ERR_ARG;
    if (pool->n_pages <= 0 || pool->max_seqs <= 0 || pool->kv_heads <= 0 || pool->kv_heads > 65535) return XSV_ERR_ARG;
    if (pool->head_dim != 64 && pool->head_dim != 128) return XSV_ERR_ARG;
    if (pool->dtype != XSV_F16 && pool->dtype != XSV_BF16) return XSV_ERR_ARG;
    if (pool->n_pages > XSV_PAGE_MAX_PAGES || pool->max_seqs > XSV_PAGE_MAX_SEQS) return XSV_ERR_LIMIT;
    if (((uintptr_t)pool->records | (uintptr_t)pool->k_tail) & 15) return XSV_ERR_SHAPE;
    *v = PoolView{(uint8_t*)pool->records, pool->k_tail, pool->n_pages, pool->max_seqs, pool->kv_heads};
    return XSV_OK;
}

extern "C" xsv_status xsv_page_append(const xsv_page_pool* pool, const void* K, const void* V, long long k_stride,
                                      long long v_stride, int n_tokens, const int* slot_map, const int* token_seq,
                                      const int* cu_new, const int* total_len, int n_seqs, void* stream) {
    Append p{};
    xsv_status s = xsv_pool_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_tokens < 0 || n_seqs <= 0 || n_seqs > pool->max_seqs) return XSV_ERR_ARG;
    if (n_tokens == 0) return XSV_OK;
    if (!K || !V || !slot_map || !token_seq || !cu_new || !total_len) return XSV_ERR_ARG;
    const long long row = (long long)pool->kv_heads * pool->head_dim;
    if (n_tokens > 1 && (k_stride < row || v_stride < row)) return XSV_ERR_ARG;
    if (((uintptr_t)K | (uintptr_t)V) & 15 || (k_stride | v_stride) & 7) return XSV_ERR_SHAPE;
    p.K = K; p.V = V; p.k_stride = k_stride; p.v_stride = v_stride;
    p.slot = slot_map; p.seq = token_seq; p.cu = cu_new; p.total = total_len;
    p.n_tokens = n_tokens; p.n_seqs = n_seqs;
    // A block looks for first tokens of pages among 32 new tokens, for one head.  Where most sequences bring a few tokens
    // (decoding) every token may be one, and a block each takes those that do not fill their page, a warp a head; a page
    // that one of them fills takes a block some 5 us, so that these are looked for among 8 tokens.  128 sequences, 8 heads of
    // 128, that way against the other: 1 token each 3.5 against 10.9 us, 4 tokens 5.5 against 5.8, 8 tokens 9.0 against 7.3.
    const bool decode = (long long)n_tokens <= 4LL * n_seqs;
    p.chunk = decode ? 8 : 32;
    const int warps = pool->head_dim / 32;
    p.few_heads = (pool->kv_heads + warps - 1) / warps;
    const long long few = decode ? (long long)n_tokens * p.few_heads : 0, blocks = few + (long long)((n_tokens + p.chunk - 1) / p.chunk) * pool->kv_heads;
    if (blocks > 0x7FFFFFFFLL) return XSV_ERR_LIMIT;
    p.few_blocks = (int)few;
    const dim3 grid((unsigned)blocks);
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, grid, dim3(pool->head_dim), 0, (cudaStream_t)stream, p); };
    cudaError_t e;
    if (pool->dtype == XSV_F16) e = pool->head_dim == 64 ? go(page_append_kernel<__half, 64>) : go(page_append_kernel<__half, 128>);
    else e = pool->head_dim == 64 ? go(page_append_kernel<__nv_bfloat16, 64>) : go(page_append_kernel<__nv_bfloat16, 128>);
    if (e != cudaSuccess) return xsv_cuda_status(e);
    xsv_count_launch(1);
    return XSV_OK;
}

extern "C" xsv_status xsv_page_read(const xsv_page_pool* pool, const int* block_table, int table_width, const int* total_len,
                                    int n_seqs, const int* token_seq, const int* positions, int n_rows, void* K_out,
                                    void* V_out, void* stream) {
    Read p{};
    xsv_status s = xsv_pool_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_rows < 0 || n_seqs <= 0 || n_seqs > pool->max_seqs || table_width <= 0) return XSV_ERR_ARG;
    if (n_rows == 0) return XSV_OK;
    if (!block_table || !total_len || !token_seq || !positions || !K_out || !V_out) return XSV_ERR_ARG;
    if (((uintptr_t)K_out | (uintptr_t)V_out) & 15) return XSV_ERR_SHAPE;
    p.table = block_table; p.total = total_len; p.seq = token_seq; p.pos = positions; p.K = K_out; p.V = V_out;
    p.width = table_width; p.n_seqs = n_seqs; p.n_rows = n_rows;
    const dim3 grid((n_rows + READ_ROWS - 1) / READ_ROWS, pool->kv_heads);
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, grid, dim3(256), 0, (cudaStream_t)stream, p); };
    cudaError_t e;
    if (pool->dtype == XSV_F16) e = pool->head_dim == 64 ? go(page_read_kernel<__half, 64>) : go(page_read_kernel<__half, 128>);
    else e = pool->head_dim == 64 ? go(page_read_kernel<__nv_bfloat16, 64>) : go(page_read_kernel<__nv_bfloat16, 128>);
    if (e != cudaSuccess) return xsv_cuda_status(e);
    xsv_count_launch(1);
    return XSV_OK;
}
