// The pages of 8-bit keys that each new token attends to: the first and the most recent ones, and of those between the best by a
// score of the token's queries against the pages' mean keys.
//
//   score(token, head, page) = max over the group's query heads of (dot * factor) * a,  dot = sum of q8 * mean codes,
//   a = max(max |q|, 2^-60),  q8 = nearest-even of q * (127 / a)
// Mean codes and q8 are whole numbers, so dot is exact (at most 127 * 127 * 128 < 2^24, a float32 too) and the score has the two
// roundings that the formula has, whatever order the sums are taken in: a selection can be repeated bit for bit.
//
// Reads d + 4 bytes a page and head where the attention reads 128 d, so what bounds it is latency for single tokens, and
// selecting (not scoring) for many.  A block takes a few tokens of one head: mma.m16n8k32 over 16 pages x 8 query rows, keys of the scores
// (unsigned, in their order) into shared memory, then the k-th largest by four histograms of 8 bits and a pass that writes
// page numbers in order.  A cluster of up to 8 blocks shares the pages of one token where few tokens have long sequences: each
// stores its scores into the first block's shared memory, which selects.
#include <algorithm>

#include "../../include/xsv.h"
#include "page8_layout.cuh"
#include "page_attn.cuh"
#include "xsv_kernels.h"

namespace {

constexpr int WARPS = 8, THREADS = WARPS * 32;

struct Select {
    PoolView pool;
    const void* Q;
    long long q_stride;
    const int* table;
    const int* seq;
    const int* pos;
    const int* slot;     // the plan's, or null
    int* out;
    int width, n_seqs, n_tokens, group, top, first, recent;
    int tokens;          // of a block
    int cols;            // query rows of a token: the group, up to a power of two below 8, else a multiple of 8
    int cluster;         // blocks that share a token's pages
};

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Unsigned numbers in the order of the floats, 0 left free (for a page that is not there).
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);               // -0 and 0 are equal
    return (b & 0x80000000u) ? max(~b, 1u) : b | 0x80000000u;
}
__host__ __device__ constexpr int query_stride(int d) { return d == 64 ? 64 : d + 64; }      // of q8 rows: neighbouring rows on different banks

// The k largest of keys[0, n) (0: not there), lowest index first among equal ones, as numbers from + index in ascending order to
// `to`; returns how many.  W warps take part, `wid` this one's number among them; hist: 256 ints, note: 2 W + 2 ints, theirs.
template <int W> __device__ __forceinline__ void together() {
    if (W == 1) __syncwarp(); else __syncthreads();
}
template <int W> __device__ int take(const uint32_t* keys, int n, int k, int from, int* to, int* hist, int* note, int wid) {
    const int lane = threadIdx.x & 31, tid = wid * 32 + lane;
    uint32_t prefix = 0u;
    int rem = k, shift = 24;
    bool all = k >= n, none = k <= 0;                          // the same for everyone
    if (!all && !none) {
        for (;; shift -= 8) {
            for (int i = tid; i < 256; i += 32 * W) hist[i] = 0;
            together<W>();
            for (int i0 = wid * 32; i0 < n; i0 += 32 * W) {
                const uint32_t key = i0 + lane < n ? keys[i0 + lane] : 0u;
                const bool in = key != 0u && (shift == 24 || key >> (shift + 8) == prefix);
                const uint32_t bin = in ? key >> shift & 255u : 256u;
                const uint32_t same = __match_any_sync(0xFFFFFFFFu, bin);
                if (in && (same & ((1u << lane) - 1u)) == 0u) atomicAdd(hist + bin, __popc(same));
            }
            together<W>();
            if (wid == 0) {                                    // lane 31 has the highest bins
                int c[8], sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) { c[i] = hist[8 * lane + i]; sum += c[i]; }
                int above = sum;                               // of this lane and those over it
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_down_sync(0xFFFFFFFFu, above, o);
                    if (lane + o < 32) above += y;
                }
                const int total = __shfl_sync(0xFFFFFFFFu, above, 0);
                above -= sum;
                if (total < rem) {                             // fewer are there than asked for (first pass only)
                    if (lane == 0) note[0] = -1;
                } else if (above < rem && above + sum >= rem) {
                    int bin = 7;
#pragma unroll
                    for (int i = 7; i >= 0; --i) {
                        if (above >= rem) continue;
                        if (above + c[i] >= rem) { bin = i; note[1] = rem - above; hist[0] = c[i]; above = rem; }
                        else above += c[i];
                    }
                    note[0] = 8 * lane + bin;
                }
            }
            together<W>();
            const int bin = note[0];
            if (bin < 0) { all = true; break; }
            rem = note[1];
            prefix = prefix << 8 | (uint32_t)bin;
            const int here = hist[0];
            together<W>();                                     // (before the histogram is cleared)
            if (shift == 0 || here == rem) break;              // the whole bin is taken
        }
    }
    if (none) return 0;
    // Every warp has a contiguous part: how many above the prefix, how many equal to it.
    const int per = (n + 32 * W - 1) / (32 * W) * 32, i0 = min(n, wid * per), i1 = min(n, i0 + per);
    auto look = [&](int i, bool& gt, bool& eq) {
        const uint32_t key = i < i1 ? keys[i] : 0u, top = key >> shift;
        gt = key != 0u && (all || top > prefix);
        eq = key != 0u && !all && top == prefix;
    };
    int n_gt = 0, n_eq = 0;
    if (W > 1) {
        for (int i = i0; i < i1; i += 32) {
            bool gt, eq;
            look(i + lane, gt, eq);
            n_gt += __popc(__ballot_sync(0xFFFFFFFFu, gt));
            n_eq += __popc(__ballot_sync(0xFFFFFFFFu, eq));
        }
        if (lane == 0) { note[2 + 2 * wid] = n_gt; note[3 + 2 * wid] = n_eq; }
        together<W>();
    }
    int eq_before = 0, at = 0;
    for (int w = 0; w < (W > 1 ? wid : 0); ++w) {
        at += note[2 + 2 * w] + min(note[3 + 2 * w], max(0, rem - eq_before));
        eq_before += note[3 + 2 * w];
    }
    for (int i = i0; i < i1; i += 32) {
        bool gt, eq;
        look(i + lane, gt, eq);
        const uint32_t below = (1u << lane) - 1u, eqs = __ballot_sync(0xFFFFFFFFu, eq);
        const bool in = gt || (eq && eq_before + __popc(eqs & below) < rem);
        const uint32_t ins = __ballot_sync(0xFFFFFFFFu, in);
        if (in) to[at + __popc(ins & below)] = from + i + lane;
        at += __popc(ins);
        eq_before += __popc(eqs);
    }
    if (W == 1) return at;
    together<W>();
    if (wid == W - 1 && lane == 0) note[0] = at;
    together<W>();
    return note[0];
}

// One token's list: the first pages, the best of those between, the most recent ones, -1.
template <int W> __device__ __forceinline__ void list_of(const Select& p, const uint32_t* keys, int mine, int* out, int* hist, int* note, int wid) {
    const int lane = threadIdx.x & 31, tid = wid * 32 + lane;
    int n = 0;
    if (mine >= 0) {
        const int nf = min(p.first, mine + 1), r0 = max(nf, mine - p.recent + 1), nr = mine + 1 - r0;      // recent: [r0, mine]
        for (int i = tid; i < nf; i += 32 * W) out[i] = i;
        const int mid = r0 - nf > 0 ? take<W>(keys + nf, r0 - nf, p.top - nf - nr, nf, out + nf, hist, note, wid) : 0;
        for (int i = tid; i < nr; i += 32 * W) out[nf + mid + i] = r0 + i;
        n = nf + mid + nr;
    }
    for (int i = n + tid; i < p.top; i += 32 * W) out[i] = -1;
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS) page8_select_kernel(const __grid_constant__ Select p) {
    using R = Page8Rec<D>;
    constexpr int KB = D / 64, QS = query_stride(D), CH = D / 32;      // CH: channels of a lane
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int s_mine[8], s_seq[8], s_hist[WARPS][256], s_note[WARPS][2 * WARPS + 2];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, j = lane & 3;
    const int cols = p.cols, rows = (p.tokens * cols + 7) / 8 * 8;
    uint8_t* const q8 = smem;                                  // [rows][QS]
    float* const qa = reinterpret_cast<float*>(smem + rows * QS);            // [rows]
    uint32_t* const keys = reinterpret_cast<uint32_t*>(qa + rows);           // [tokens][width]
    const int rank = blockIdx.x % p.cluster, unit = blockIdx.x / p.cluster, head = unit % p.pool.heads, t0 = unit / p.pool.heads * p.tokens;
    const int here = min(p.tokens, p.n_tokens - t0);
    if (p.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    xsv_dep_release();
    xsv_dep_sync();
    // ---- tokens; -1: one that selects nothing
    if (tid < p.tokens) {
        int mine = -1, seq = -1;
        if (tid < here) {
            seq = p.seq[t0 + tid];
            const int pos = p.pos[t0 + tid];
            if (seq >= 0 && seq < p.n_seqs && pos >= 0 && !(p.slot && p.slot[t0 + tid] < 0)) mine = min(pos / XSV_PAGE, p.width - 1);
        }
        s_mine[tid] = mine;
        s_seq[tid] = seq;
    }
    // ---- queries -> q8: a warp a row; rows beyond the group repeat its first head, which changes no maximum
    for (int r = wid; r < rows; r += WARPS) {
        const int i = r / cols, c = r - i * cols, h = head * p.group + (c < p.group ? c : 0);
        float x[CH], a = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) x[k] = 0.f;
        if (i < here) {
            const T* src = (const T*)p.Q + (size_t)(t0 + i) * p.q_stride + (size_t)h * D + CH * lane;
#pragma unroll
            for (int k = 0; k < CH; k += 2) {
                const float2 f = xsv_unpack2<T>(*reinterpret_cast<const uint32_t*>(src + k));
                x[k] = f.x; x[k + 1] = f.y;
                a = fmaxf(a, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
        }
        a = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(a)));
        a = fmaxf(a, 8.67361737988403547e-19f);                // 2^-60
        const float inv = __fdiv_rn(127.f, a);
        uint32_t w = 0;
#pragma unroll
        for (int k = 0; k < CH; ++k) w |= ((uint32_t)__float2int_rn(__fmul_rn(x[k], inv)) & 0xFFu) << (8 * k);
        if (CH == 4) *reinterpret_cast<uint32_t*>(q8 + r * QS + 4 * lane) = w;
        else *reinterpret_cast<unsigned short*>(q8 + r * QS + 2 * lane) = (unsigned short)w;
        if (lane == 0) qa[r] = a;
    }
    uint32_t lead = smem_u32(keys);                            // the first block's keys
    if (p.cluster > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");          // all blocks run: their shared memory can be written
        asm("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(lead));
    }
    __syncthreads();
    auto store = [&](int i, int page, uint32_t key) {
        const uint32_t at = lead + 4u * (uint32_t)(i * p.width + page);
        if (p.cluster > 1) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(key) : "memory");
        else keys[i * p.width + page] = key;
    };
    // ---- scores: runs of tokens of one sequence, 16 pages a warp at a time
    for (int a = 0; a < here;) {
        int b = a + 1, far = s_mine[a];
        while (b < here && s_seq[b] == s_seq[a]) far = max(far, s_mine[b++]);
        const int* row = p.table + (size_t)max(s_seq[a], 0) * p.width;
        const int end = far - p.recent + 1;                    // pages [first, end) may be scored (far < 0: none)
        for (int base = p.first + (rank * WARPS + wid) * 16; base < end; base += p.cluster * WARPS * 16) {
            const uint8_t* rec[2];
            uint4 m[2][KB];
            float f[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int page = base + g + 8 * u, id = page < end ? row[page] : -1;
                const bool there = (unsigned long long)(long long)id < (unsigned long long)p.pool.n_pages;
                rec[u] = there ? page8_rec<D>(p.pool, id, head) : nullptr;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f[u] = 0.f;
#pragma unroll
                for (int c = 0; c < KB; ++c) m[u][c] = make_uint4(0u, 0u, 0u, 0u);
                if (rec[u]) {
#pragma unroll
                    for (int c = 0; c < KB; ++c) m[u][c] = *reinterpret_cast<const uint4*>(rec[u] + R::MEAN + 64 * c + 16 * j);
                    f[u] = reinterpret_cast<const float*>(rec[u] + R::PARAMS)[2];
                }
            }
            float best[2][2];                                  // [page][token of the lane's columns, where they are two]
            for (int n = a * cols / 8; n < (b * cols + 7) / 8; ++n) {
                int c[4] = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    const uint4 q = *reinterpret_cast<const uint4*>(q8 + (8 * n + g) * QS + 64 * k + 16 * j);
                    mma_s8(c, m[0][k].x, m[1][k].x, m[0][k].y, m[1][k].y, q.x, q.y);
                    mma_s8(c, m[0][k].z, m[1][k].z, m[0][k].w, m[1][k].w, q.z, q.w);
                }
                const float2 a2 = *reinterpret_cast<const float2*>(qa + 8 * n + 2 * j);
                float s[2][2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    s[u][0] = __fmul_rn(__fmul_rn((float)c[2 * u], f[u]), a2.x);
                    s[u][1] = __fmul_rn(__fmul_rn((float)c[2 * u + 1], f[u]), a2.y);
                    if (cols > 1) s[u][0] = fmaxf(s[u][0], s[u][1]);
                    if (cols > 2) s[u][0] = fmaxf(s[u][0], __shfl_xor_sync(0xFFFFFFFFu, s[u][0], 1));
                    if (cols > 4) s[u][0] = fmaxf(s[u][0], __shfl_xor_sync(0xFFFFFFFFu, s[u][0], 2));
                }
                if (cols > 8) {                                // a token's rows are several tiles
                    const bool begins = n * 8 % cols == 0;
#pragma unroll
                    for (int u = 0; u < 2; ++u) best[u][0] = begins ? s[u][0] : fmaxf(best[u][0], s[u][0]);
                    if ((n + 1) * 8 % cols != 0) continue;
#pragma unroll
                    for (int u = 0; u < 2; ++u) s[u][0] = best[u][0];
                }
                // one lane stores a token's score: the first of those that have it
                const int col = 8 * n + 2 * j;
                const bool mine = cols <= 2 || (cols == 4 ? (j & 1) == 0 : j == 0);
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    if (!mine || (v == 1 && cols > 1)) continue;
                    const int i = (col + v) / cols;
                    if (i < a || i >= b) continue;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int page = base + g + 8 * u;
                        if (page < end) store(i, page, rec[u] ? order_of(s[u][v]) : 0u);
                    }
                }
            }
        }
        a = b;
    }
    if (p.cluster > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank != 0) return;
    }
    __syncthreads();
    // ---- the lists
    if (p.tokens == 1) {
        list_of<WARPS>(p, keys, s_mine[0], p.out + ((size_t)t0 * p.pool.heads + head) * p.top, s_hist[0], s_note[0], wid);
        return;
    }
    for (int i = wid; i < here; i += WARPS)
        list_of<1>(p, keys + (size_t)i * p.width, s_mine[i], p.out + ((size_t)(t0 + i) * p.pool.heads + head) * p.top, s_hist[wid], s_note[wid], 0);
}

size_t smem_of(int tokens, int cols, int head_dim, int width) {
    const int rows = (tokens * cols + 7) / 8 * 8;
    return (size_t)rows * (query_stride(head_dim) + 4) + (size_t)tokens * width * 4;
}
constexpr size_t SMEM_MAX = 200 * 1024;

template <typename T, int D> cudaError_t launch(const Select& p, long long blocks, cudaStream_t st) {
    auto kernel = page8_select_kernel<T, D>;
    static XsvPerDeviceInt ready;
    const int dev = xsv_current_device();
    if (!ready.get(dev)) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_MAX);
        if (e != cudaSuccess) return e;
        ready.set(dev, 1);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem_of(p.tokens, p.cols, D, p.width);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (p.cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)p.cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (xsv_dep_launch_enabled()) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e == cudaSuccess) xsv_count_launch(1);
    return e;
}

}  // namespace

extern "C" xsv_status xsv_page8_select(const xsv_page8_pool* pool, const void* Q, long long q_stride, int n_tokens, int q_heads, const int* block_table,
                                       int table_width, int n_seqs, const int* token_seq, const int* positions, const int* slot_map, int top, int first,
                                       int recent, int* selected, void* stream) {
    Select p{};
    xsv_status s = xsv_page8_view(pool, &p.pool);
    if (s != XSV_OK) return s;
    if (n_tokens < 0 || n_seqs <= 0 || n_seqs > XSV_PAGE_MAX_SEQS || table_width <= 0) return XSV_ERR_ARG;
    if (q_heads < pool->kv_heads || q_heads % pool->kv_heads) return XSV_ERR_ARG;
    if (top <= 0 || first < 0 || recent < 1 || first > top - recent) return XSV_ERR_ARG;
    if (n_tokens == 0) return XSV_OK;
    if (!Q || !block_table || !token_seq || !positions || !selected) return XSV_ERR_ARG;
    if (n_tokens > 1 && q_stride < (long long)q_heads * pool->head_dim) return XSV_ERR_ARG;
    if ((uintptr_t)Q & 15 || q_stride & 7) return XSV_ERR_SHAPE;
    p.group = q_heads / pool->kv_heads;
    if (p.group > XSV_PAGE8_MAX_GROUP || table_width > XSV_PAGE8_MAX_WIDTH || top > XSV_PAGE8_MAX_TOP) return XSV_ERR_LIMIT;
    p.Q = Q; p.q_stride = q_stride; p.table = block_table; p.seq = token_seq; p.pos = positions; p.slot = slot_map; p.out = selected;
    p.width = table_width; p.n_seqs = n_seqs; p.n_tokens = n_tokens; p.top = top; p.first = first; p.recent = recent;
    p.cols = p.group >= 8 ? (p.group + 7) / 8 * 8 : p.group > 4 ? 8 : p.group > 2 ? 4 : p.group;
    // Many tokens: 8 a block, a warp selects for each; few: one, and up to 8 blocks a token while there are idle
    // multiprocessors and each block has 128 pages at least.
    const long long units = (long long)n_tokens * pool->kv_heads;
    p.tokens = 1;
    p.cluster = 1;
    if (units >= 8LL * 2 * xsv_sm_count()) {
        p.tokens = 8;
        while (p.tokens > 1 && (smem_of(p.tokens, p.cols, pool->head_dim, table_width) > SMEM_MAX || p.tokens * p.cols > XSV_PAGE8_MAX_GROUP)) p.tokens /= 2;
    } else {
        while (p.cluster < 8 && units * p.cluster * 2 <= 2 * xsv_sm_count() && table_width >= 256 * p.cluster) p.cluster *= 2;
    }
    const long long blocks = ((long long)n_tokens + p.tokens - 1) / p.tokens * pool->kv_heads * p.cluster;
    if (blocks > 0x7FFFFFFFLL) return XSV_ERR_LIMIT;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (pool->dtype == XSV_F16) e = pool->head_dim == 64 ? launch<__half, 64>(p, blocks, st) : launch<__half, 128>(p, blocks, st);
    else e = pool->head_dim == 64 ? launch<__nv_bfloat16, 64>(p, blocks, st) : launch<__nv_bfloat16, 128>(p, blocks, st);
    return e == cudaSuccess ? XSV_OK : xsv_cuda_status(e);
}
