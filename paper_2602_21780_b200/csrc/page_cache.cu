// Writing the pages of the shared pool, and reading them back as values.
//
// xsv_page_append: one block per (new tokens of one page, head).  Values are quantised per token over 64 channels as
// they come and merged into the page's code words (a token is one byte of each word it touches); keys need all 64
// tokens of a page for their per-channel scale, so a page's keys wait in the sequence's tail, in 16 bits, and are
// quantised by the call that brings the page's last token.  The tail has two halves, by the page's parity: the page
// that is completed is read from one while the page after it starts in the other.  Bound by HBM for prompts (2 bytes
// read, 72/128 written per element); the thread layout makes both packings local to a thread -- a thread's 8 rows x
// 8 channels of keys (rows 8 i + g) are whole code words, and so are 4 tokens x 8 channels of values -- so codes never
// pass through shared memory, only the column minima and maxima do.
//
// xsv_page_read: one block per (32 listed tokens, head); a thread decodes 8 channels of one token, so that a page's
// record is fetched once into L1 for the rows that share its sectors and the outputs are written 16 bytes a thread.
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
    int n_tokens, n_seqs, chunk;
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

template <typename T, int D>
__global__ void __launch_bounds__(D, D == 128 ? 5 : 10) page_append_kernel(const __grid_constant__ Append p) {
    using R = PageRec<D>;
    constexpr int C = D / 8;                 // 8-channel pieces of a row
    __shared__ uint32_t s_mn[8][D / 2], s_mx[8][D / 2];
    __shared__ float s_scale[D], s_zero[D], s_inv[D];
    xsv_dep_release();
    xsv_dep_sync();
    const int tid = threadIdx.x, piece = tid % C, g = tid / C, head = blockIdx.y, lane = tid & 31;
    // the chunk's tokens that are the first new ones of their page; every warp finds the same
    Place mine{};
    bool first = false;
    const int t_lane = blockIdx.x * p.chunk + lane;
    if (lane < p.chunk && t_lane < p.n_tokens) first = place_of(p, t_lane, mine) && (t_lane == mine.begin || mine.off == 0);
    for (uint32_t todo = __ballot_sync(0xFFFFFFFFu, first); todo; todo &= todo - 1) {
        const int from = __ffs(todo) - 1, t = blockIdx.x * p.chunk + from;
        Place q;
        q.seq = __shfl_sync(0xFFFFFFFFu, mine.seq, from);
        q.begin = __shfl_sync(0xFFFFFFFFu, mine.begin, from);
        q.end = __shfl_sync(0xFFFFFFFFu, mine.end, from);
        q.page = __shfl_sync(0xFFFFFFFFu, mine.page, from);
        q.off = __shfl_sync(0xFFFFFFFFu, mine.off, from);
        q.pos = __shfl_sync(0xFFFFFFFFu, mine.pos, from);
        const int run = min(XSV_PAGE - q.off, q.end - t), total = q.pos + q.end - t;
        const bool full = q.off + run == XSV_PAGE;
        uint8_t* rec = page_rec<D>(p.pool, q.page, head);
        const T* K = (const T*)p.K + (size_t)head * D + 8 * piece;
        const T* V = (const T*)p.V + (size_t)head * D + 8 * piece;
        const int page_no = q.pos / XSV_PAGE;
        // The last, unfilled page's keys go to the tail half of its parity.  Where the sequence's first page here still
        // reads old keys from that half, the block of that first page writes them, after its reads.
        const int p0 = q.pos - (t - q.begin), first_no = p0 / XSV_PAGE, last_no = total / XSV_PAGE;
        const bool handed = p0 % XSV_PAGE != 0 && last_no > first_no && ((last_no - first_no) & 1) == 0;

        // ---- values: 4 tokens x 8 channels a thread, twice
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const int combo = g + 8 * half, tok0 = 16 * (combo >> 2) + 2 * (combo & 3);
            uint4 raw[4];
            bool there[4];
            uint32_t mask = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int tok = tok0 + 8 * (b & 1) + (b >> 1);
                there[b] = tok >= q.off && tok < q.off + run;
                raw[b] = make_uint4(0, 0, 0, 0);
                if (there[b]) {
                    raw[b] = *reinterpret_cast<const uint4*>(V + (size_t)(t + tok - q.off) * p.v_stride);
                    mask |= 0xFFu << (8 * b);
                }
            }
            if (!__any_sync(0xFFFFFFFFu, mask != 0)) continue;
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int tok = tok0 + 8 * (b & 1) + (b >> 1);
                float mn, mx;
                {
                    const float2 lo = xsv_unpack2<T>(min2<T>(min2<T>(raw[b].x, raw[b].y), min2<T>(raw[b].z, raw[b].w)));
                    const float2 hi = xsv_unpack2<T>(max2<T>(max2<T>(raw[b].x, raw[b].y), max2<T>(raw[b].z, raw[b].w)));
                    mn = fminf(lo.x, lo.y);
                    mx = fmaxf(hi.x, hi.y);
                }
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) {               // the 8 pieces of 64 channels are 8 neighbouring lanes
                    mn = fminf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, o));
                    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
                }
                __half hs, hz;
                page_params(clamp_half(mn), clamp_half(mx), hs, hz);
                const float s = __half2float(hs), z = __half2float(hz), inv = __frcp_rn(s);
                float x[8], near = 0.f;
                unpack8<T>(raw[b], x);
                uint32_t c[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) c[i] = code_bits(clamp_half(x[i]), inv, z, near);
                if (near > CODE_NEAR)
#pragma unroll
                    for (int i = 0; i < 8; ++i) c[i] = code_bits_exact(clamp_half(x[i]), s, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i >> 1] += (c[i] - CODE_BASE) << (8 * b + 4 * (i & 1));
                if (there[b] && piece % 8 == 0) {
                    const int at = (piece / 8) * 64 + (tok % 8) * 8 + tok / 8;
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

        // ---- keys
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
            s_scale[2 * tid] = __half2float(s0); s_scale[2 * tid + 1] = __half2float(s1);
            s_zero[2 * tid] = __half2float(z0); s_zero[2 * tid + 1] = __half2float(z1);
            s_inv[2 * tid] = __frcp_rn(__half2float(s0)); s_inv[2 * tid + 1] = __frcp_rn(__half2float(s1));
        }
        __syncthreads();
        {
            // channel c of the piece: step 2 (piece / 4) + c / 4, byte 2 (c % 2) + (c % 4) / 2; row 8 i + g: word i / 2,
            // nibble i % 2
#pragma unroll
            for (int kl = 0; kl < 2; ++kl) {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int c4 = 0; c4 < 4; ++c4) {
                    const int c = 4 * kl + c4, sh = 8 * (2 * (c % 2) + (c % 4) / 2);
                    const float s = s_scale[8 * piece + c], z = s_zero[8 * piece + c], inv = s_inv[8 * piece + c];
                    float x[8], near = 0.f;
                    uint32_t code[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t pair = c < 2 ? row[i].x : c < 4 ? row[i].y : c < 6 ? row[i].z : row[i].w;
                        const float2 two = xsv_unpack2<T>(pair);
                        x[i] = clamp_half(c & 1 ? two.y : two.x);
                        code[i] = code_bits(x[i], inv, z, near);
                    }
                    if (near > CODE_NEAR)
#pragma unroll
                        for (int i = 0; i < 8; ++i) code[i] = code_bits_exact(x[i], s, z);
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i / 2] += (code[i] - CODE_BASE) << (sh + 4 * (i % 2));
                }
                *reinterpret_cast<uint4*>(rec + R::K_CODES + ((2 * (piece / 4) + kl) * 32 + g * 4 + piece % 4) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        if (handed && page_no == first_no) {                    // after the barriers: the old keys have been read
            const int left = total % XSV_PAGE;
            T* tail = tail_rows<T, D>(p.pool, q.seq, last_no, head) + 8 * piece;
            for (int r = g; r < left; r += 8)
                *reinterpret_cast<uint4*>(tail + (size_t)r * D) = *reinterpret_cast<const uint4*>(K + (size_t)(q.end - left + r) * p.k_stride);
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
// the low four bits as a float, without the conversion unit
__device__ __forceinline__ float small(uint32_t w) { return __fadd_rn(__uint_as_float((w & 15u) | 0x4B000000u), -8388608.f); }

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
                const uint4 sc = *reinterpret_cast<const uint4*>(rec + R::K_SCALE + 16 * piece);
                const uint4 ze = *reinterpret_cast<const uint4*>(rec + R::K_ZERO + 16 * piece);
                float s[8], z[8], x[8];
                unpack8<__half>(sc, s);
                unpack8<__half>(ze, z);
#pragma unroll
                for (int kl = 0; kl < 2; ++kl) {
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(rec + R::K_CODES + ((2 * (piece / 4) + kl) * 32 + g * 4 + piece % 4) * 16 + (tok / 16) * 4) >> (4 * (tok / 8 % 2));
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[4 * kl + c] = fmaf(small(w >> (8 * (2 * (c % 2) + c / 2))), s[4 * kl + c], z[4 * kl + c]);
                }
                k = make_uint4(xsv_pack2<T>(x[0], x[1]), xsv_pack2<T>(x[2], x[3]), xsv_pack2<T>(x[4], x[5]), xsv_pack2<T>(x[6], x[7]));
            }
            const int at = (piece / 8) * 64 + g * 8 + tok / 8;
            const float s = __half2float(reinterpret_cast<const __half*>(rec + R::V_SCALE)[at]);
            const float z = __half2float(reinterpret_cast<const __half*>(rec + R::V_ZERO)[at]);
            const uint4 w = *reinterpret_cast<const uint4*>(rec + R::V_CODES + (((tok / 16) * (D / 64) + piece / 8) * 32 + (piece % 8) * 4 + tok % 8 / 2) * 16);
            const int sh = 8 * (2 * (tok % 2) + tok / 8 % 2);
            auto val = [&](uint32_t word, int i) { return fmaf(small(word >> (sh + 4 * i)), s, z); };
            v = make_uint4(xsv_pack2<T>(val(w.x, 0), val(w.x, 1)), xsv_pack2<T>(val(w.y, 0), val(w.y, 1)),
                           xsv_pack2<T>(val(w.z, 0), val(w.z, 1)), xsv_pack2<T>(val(w.w, 0), val(w.w, 1)));
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
    // A block looks for first tokens of pages among `chunk` new tokens: one each where most sequences bring a few
    // tokens (every token may be one), 16 where prompts do (one in 64 is one).
    p.chunk = (long long)n_tokens <= 8LL * n_seqs ? 1 : 16;
    const dim3 grid((n_tokens + p.chunk - 1) / p.chunk, pool->kv_heads);
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
