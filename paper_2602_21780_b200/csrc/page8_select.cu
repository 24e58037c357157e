// The pages of 8-bit keys that each new token attends to: the first and the most recent ones, and of those between the best by a
// score of the token's queries against the pages' mean keys.
//
//   score(token, head, page) = max over the group's query heads of (dot * factor) * a,  dot = sum of q8 * mean codes,
//   a = max(max |q|, 2^-60),  q8 = nearest-even of q * (127 / a)
// Mean codes and q8 are whole numbers, so dot is exact (at most 127 * 127 * 128 < 2^24, a float32 too) and the score has the two
// roundings that the formula has, whatever order the sums are taken in: a selection can be repeated bit for bit.
//
// Reads d + 4 bytes a page and head where the attention reads 128 d, so what bounds it is latency for single tokens, and
// instructions for many.  A block takes a token, or a few, of one head: mma.m16n8k32 over 16 query rows x 8 pages, the scores as unsigned
// numbers in their order ("keys") into shared memory, then the k-th largest by bracketing and a pass that writes page numbers in order.
// A cluster of up to 8 blocks shares the pages of one token where few tokens have long sequences: each stores its keys into the first block's
// shared memory, which selects.
//
// The first and the recent pages are looked up in the table at the start, beside the scores' loads, since one that is not there is not
// listed and leaves its place to another.
//
// Measured.  32 query and 8 key/value heads of 128, 32 pages each: 16 tokens over 2000 to 60 000: 11.5 us, of which the launch and
// four loads that wait for one another (token, table, mean key; query) are about 6, the selection 3; 1021 tokens over 40 000: 41 us, half of it
// the scores' and half of it the selections' instructions, at 32 warps a multiprocessor (at 16: 50).
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
    int rows;            // query rows of a token: the group, up to a power of two below 16, else a multiple of 16
    int cluster;         // blocks that share a token's pages
};

// d = a b + c for all of d the same
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, int c) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(c));
}
__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Unsigned numbers in the order of the floats, 0 left free (for a page that is not there), and back.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);               // -0 and 0 are equal
    return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k ^ ((uint32_t)((int)~k >> 31) | 0x80000000u)); }
__device__ __forceinline__ unsigned long long f2_mul(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
constexpr int MAGIC = 0x4B400000;                              // the float 1.5 * 2^23: plus a whole number below 2^22, as bits or as floats
__host__ __device__ constexpr int key_stride(int width) { return (width + 31) / 32 * 32 + 32; }

// The k largest of keys[0, n) (0: not there), lowest index first among equal ones, as numbers from + index in ascending order to
// `to`; returns how many.  W warps take part, `wid` this one's number among them; note: 6 W + 1 ints of theirs.  A lane holds N keys in
// registers (N 0: any number, read again from shared memory for every step).
//
// The k-th largest is found by bracketing: between the least and the largest key, as the floats that they stand for, by turns
// where the logarithm of the number of keys above would reach log k if it were linear in the score (the upper ends of
// distributions nearly are) and in the middle, and after 40 steps as whole numbers, which ends for certain; as soon as
// exactly k keys are above it is done.  Counting costs a comparison and an addition a key, and no two lanes write to the same place, as
// they would in a histogram of the scores' leading bits (1021 tokens over 620 pages: 81 us with four histograms of 8 bits).
template <int W> __device__ __forceinline__ void together() {
    if (W == 1) __syncwarp(); else __syncthreads();
}
template <int W, int N> __device__ __noinline__ int take(const uint32_t* keys, int n, int k, int from, int* to, int* note, int wid) {
    const int lane = threadIdx.x & 31;
    constexpr int HELD = N > 0 ? N : 1;
    // every warp has a contiguous part
    const int per = N > 0 ? 32 * N : (n + 32 * W - 1) / (32 * W) * 32, i0 = min(n, wid * per), i1 = min(n, i0 + per);
    uint32_t key[HELD];
    if (N > 0) {
#pragma unroll
        for (int r = 0; r < HELD; ++r) key[r] = i0 + 32 * r + lane < i1 ? keys[i0 + 32 * r + lane] : 0u;
    }
    auto each = [&](auto f) {                                  // f(key), whole warps
        if (N > 0) {
#pragma unroll
            for (int r = 0; r < HELD; ++r) f(key[r]);
        } else {
#pragma unroll 4
            for (int i = i0; i < i1; i += 32) f(i + lane < i1 ? keys[i + lane] : 0u);
        }
    };
    // a number summed over the warps (two buffers, so that one barrier a sum is enough)
    int turn = 0;
    auto sum = [&](int c) {
        c = __reduce_add_sync(0xFFFFFFFFu, c);
        if (W == 1) return c;
        if (lane == 0) note[turn * W + wid] = c;
        together<W>();
        c = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) c += note[turn * W + w];
        turn ^= 1;
        return c;
    };
    uint32_t least = 0xFFFFFFFFu, most = 0u;
    int c = 0;
    each([&](uint32_t x) {
        c += x != 0u ? 1 : 0;
        least = min(least, x - 1u);                            // (0 is not among them)
        most = max(most, x);
    });
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    if (W > 1) {
        if (lane == 0) { note[2 * W + wid] = (int)least; note[3 * W + wid] = (int)most; }
        c = sum(c);
#pragma unroll
        for (int w = 0; w < W; ++w) { least = min(least, (uint32_t)note[2 * W + w]); most = max(most, (uint32_t)note[3 * W + w]); }
    } else {
        c = sum(c);
    }
    uint32_t lo = 1u;                                          // the k-th largest, in the end; all that are there, if they are no more
    int rem = n;                                               // of those equal to lo that are taken
    if (c > k) {
        uint32_t hi = most;
        int c_lo = c, c_hi = 0;                                // keys >= lo: more than k; keys > hi: fewer
        lo = least + 1u;
        const float log_k = __log2f((float)k + 0.5f);
        for (int step = 0; lo < hi; ++step) {
            uint32_t mid = lo + ((hi - lo) >> 1) + 1u;
            if (step < 40) {
                float part = 0.5f;
                if ((step & 1) == 0) {
                    const float l = __log2f((float)c_lo), h = __log2f(fmaxf((float)c_hi, 0.5f));
                    part = __fdividef(l - log_k, l - h);
                }
                const float x = value_of(lo);
                mid = order_of(x + part * (value_of(hi) - x));
            }
            mid = min(max(mid, lo + 1u), hi);
            c = 0;
            // x >= mid where x + (2^32 - mid) carries; two counters, one after the other
            int other = 0;
            each([&](uint32_t x) {
                asm("{\n\t.reg .u32 t;\n\tadd.cc.u32 t, %1, %2;\n\taddc.u32 %0, %0, 0;\n\t}" : "+r"(c) : "r"(x), "r"(0u - mid));
                const int y = c;
                c = other;
                other = y;
            });
            c = sum(c + other);
            if (c >= k) { lo = mid; c_lo = c; }
            if (c == k) break;
            if (c < k) { hi = mid - 1u; c_hi = c; }
        }
        if (c_lo > k) rem = k - c_hi;                          // (else all that are equal to lo)
    }
    const bool ties = rem < n;                                 // the same for everyone
    int eq_before = 0, at = 0;
    if (W > 1) {
        int n_gt = 0, n_eq = 0;
        each([&](uint32_t x) {
            n_gt += x > lo ? 1 : 0;
            n_eq += x == lo ? 1 : 0;
        });
        n_gt = __reduce_add_sync(0xFFFFFFFFu, n_gt);
        n_eq = __reduce_add_sync(0xFFFFFFFFu, n_eq);
        if (lane == 0) { note[4 * W + wid] = n_gt; note[5 * W + wid] = n_eq; }
        together<W>();
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w >= wid) break;
            at += note[4 * W + w] + min(note[5 * W + w], max(0, rem - eq_before));
            eq_before += note[5 * W + w];
        }
    }
    const uint32_t below = (1u << lane) - 1u;
    int i = from + i0 + lane;
    each([&](uint32_t x) {
        bool in = x >= lo;
        if (ties) {
            const uint32_t eqs = __ballot_sync(0xFFFFFFFFu, x == lo);
            in = x > lo || (x == lo && eq_before + __popc(eqs & below) < rem);
            eq_before += __popc(eqs);
        }
        const uint32_t ins = __ballot_sync(0xFFFFFFFFu, in);
        if (in) to[at + __popc(ins & below)] = i;
        at += __popc(ins);
        i += 32;
    });
    if (W == 1) return at;
    if (wid == W - 1 && lane == 0) note[6 * W] = at;
    together<W>();
    return note[6 * W];
}
template <int W> __device__ __forceinline__ int take_any(const uint32_t* keys, int n, int k, int from, int* to, int* note, int wid) {
    if (k <= 0 || n <= 0) return 0;
    if (n <= 32 * W * (W == 1 ? 8 : 2)) return take<W, W == 1 ? 8 : 2>(keys, n, k, from, to, note, wid);
    if (n <= 32 * W * (W == 1 ? 20 : 4)) return take<W, W == 1 ? 20 : 4>(keys, n, k, from, to, note, wid);
    if (n <= 32 * W * (W == 1 ? 32 : 12)) return take<W, W == 1 ? 32 : 12>(keys, n, k, from, to, note, wid);
    return take<W, 0>(keys, n, k, from, to, note, wid);
}

// The pages that a token whose own page is `mine` takes unscored if the table has them: the first nf, and those from r0 on.
struct Fixed {
    int nf, r0, n;
    __device__ __forceinline__ Fixed(const Select& p, int mine) : nf(min(p.first, mine + 1)), r0(max(nf, mine - p.recent + 1)), n(nf + mine + 1 - r0) {}
    __device__ __forceinline__ int page(int x) const { return x < nf ? x : r0 + x - nf; }
};
// The place of the x-th of them, -1 beyond the last.
__device__ __forceinline__ int fixed_place(const Select& p, const Fixed& f, int seq, int x) { return x < f.n ? p.table[(size_t)seq * p.width + f.page(x)] : -1; }

// One token's list: the first pages, the best of those between, the most recent ones, -1.  ahead: fixed_place of this lane, looked up before.
template <int W> __device__ __forceinline__ void list_of(const Select& p, const uint32_t* keys, int seq, int mine, int ahead, int* out, int* note, int wid) {
    const int lane = threadIdx.x & 31, tid = wid * 32 + lane;
    int n = 0;
    if (mine >= 0) {
        const Fixed f(p, mine);
        auto there = [&](int x0) {                             // of the 32 from x0 on
            const int page = x0 == 0 ? ahead : fixed_place(p, f, seq, x0 + lane);
            return __ballot_sync(0xFFFFFFFFu, (unsigned long long)(long long)page < (unsigned long long)p.pool.n_pages);
        };
        int has = 0, has_first = 0;
        for (int x0 = 0; x0 < f.n; x0 += 32) {
            const uint32_t in = there(x0);
            has += __popc(in);
            if (x0 < f.nf) has_first += __popc(f.nf - x0 < 32 ? in & ((1u << (f.nf - x0)) - 1u) : in);
        }
        const int mid = take_any<W>(keys + f.nf, f.r0 - f.nf, p.top - has, f.nf, out + has_first, note, wid);
        n = has + mid;
        if (wid == 0) {
            int at = 0;
            for (int x0 = 0; x0 < f.n; x0 += 32) {
                const uint32_t in = there(x0);
                const int x = x0 + lane;
                if (in >> lane & 1u) out[at + __popc(in & ((1u << lane) - 1u)) + (x < f.nf ? 0 : mid)] = f.page(x);
                at += __popc(in);
            }
        }
    }
    for (int i = n + tid; i < p.top; i += 32 * W) out[i] = -1;
}

// ROWS: query rows of a token in a tile of 16 (16: it has p.rows / 16 tiles); MODE: see there.
// The queries are the 16-row operand, pages the 8 columns: a lane's 16 bytes of a mean key are two register pairs of that operand as
// they come, and the queries' registers are put together once, when they are quantised.  Row g of a tile and row g + 8 are neighbouring heads
// of a token, so that the first step of the maximum over its heads needs no exchange.
template <int ROWS> __device__ __forceinline__ void row_place(int rr, int& token, int& head) {
    const int g = rr & 7, high = rr >> 3;
    if constexpr (ROWS == 1) {
        token = rr;
        head = 0;
    } else {
        token = g / (ROWS / 2);
        head = g % (ROWS / 2) * 2 + high;
    }
}

// Many tokens: 16 pages a warp and turn instead of 32, so that registers for 32 warps a multiprocessor remain.
enum Mode { ONE, SHARED, MANY };                               // a token a block, a token a cluster of blocks, 8 tokens a block

template <typename T, int D, int ROWS, Mode MODE>
__global__ void __launch_bounds__(THREADS, MODE == MANY ? 4 : 2) page8_select_kernel(const __grid_constant__ Select p) {
    using R = Page8Rec<D>;
    constexpr bool CLUSTER = MODE == SHARED;
    constexpr int KB = D / 64, CH = D / 32, TOKENS = 16 / ROWS, NU = MODE == MANY ? 2 : 4, TURN = 8 * NU;              // CH: channels of a lane; TOKENS: of a tile
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int s_mine[8], s_seq[8], s_note[6 * WARPS + 1];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, j = lane & 3;
    const int each = ROWS < 16 ? 1 : p.rows / 16, tiles = ROWS < 16 ? (p.tokens + TOKENS - 1) / TOKENS : p.tokens * each, across = key_stride(p.width);
    uint8_t* const q8 = smem;                                  // [tiles][2 KB steps][32 lanes][4 registers] words of 4 channels
    float* const qa = reinterpret_cast<float*>(smem + tiles * 16 * D);       // [tiles][16]
    uint32_t* const keys = reinterpret_cast<uint32_t*>(qa + tiles * 16);     // [tokens][across]
    const int rank = CLUSTER ? blockIdx.x % p.cluster : 0, unit = CLUSTER ? blockIdx.x / p.cluster : blockIdx.x, head = unit % p.pool.heads,
              t0 = unit / p.pool.heads * p.tokens;
    const int here = min(p.tokens, p.n_tokens - t0);
    if (CLUSTER) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
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
    __syncthreads();
    // ---- pages: TURN a warp at a time, of a run of tokens of one sequence
    uint4 m[NU][KB];                                           // mean keys of pages 8 u + g, channels 64 c + 16 j to + 15
    float f[NU];
    uint32_t there = 0;                                        // bit u
    int run = 0, end = 0;                                      // the run's end; its pages [first, end) may be scored
    auto begin_run = [&](int a) {
        int far = s_mine[a];
        for (run = a + 1; run < here && s_seq[run] == s_seq[a];) far = max(far, s_mine[run++]);
        end = far - p.recent + 1;                              // (far < 0: none)
    };
    auto look_up = [&](int a, int base) { return lane < TURN && base + lane < end ? p.table[(size_t)max(s_seq[a], 0) * p.width + base + lane] : -1; };
    auto fetch = [&](int id) {
        there = 0;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int page = __shfl_sync(0xFFFFFFFFu, id, 8 * u + g);
            const bool is = (unsigned long long)(long long)page < (unsigned long long)p.pool.n_pages;
            there |= (is ? 1u : 0u) << u;
            f[u] = 0.f;
#pragma unroll
            for (int c = 0; c < KB; ++c) m[u][c] = make_uint4(0u, 0u, 0u, 0u);
            if (is) {
                const uint8_t* rec = page8_rec<D>(p.pool, page, head);
#pragma unroll
                for (int c = 0; c < KB; ++c) m[u][c] = *reinterpret_cast<const uint4*>(rec + R::MEAN + 64 * c + 16 * j);
                f[u] = reinterpret_cast<const float*>(rec + R::PARAMS)[2];
            }
        }
    };
    // (a warp's token is its number where a block has several, 8 at most)
    const int listed = MODE == MANY ? wid : 0;
    int ahead = -1;
    if (listed < here && s_mine[listed] >= 0) ahead = fixed_place(p, Fixed(p, s_mine[listed]), s_seq[listed], lane);
    const int base0 = p.first + (rank * WARPS + wid) * TURN, step = (CLUSTER ? p.cluster : 1) * WARPS * TURN;
    begin_run(0);
    if (base0 < end) fetch(look_up(0, base0));                 // on their way while the queries are read
    // ---- queries -> q8: a warp a row; rows beyond the group repeat its first head, which changes no maximum
    constexpr int AHEAD = 4;                                   // rows of a warp whose loads are on their way together
    for (int r0 = wid; r0 < tiles * 16; r0 += AHEAD * WARPS) {
        uint32_t raw[AHEAD][CH / 2];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const int r = r0 + e * WARPS;
            int i, h;
            row_place<ROWS>(r & 15, i, h);
            if (ROWS < 16) {
                i += (r >> 4) * TOKENS;
            } else {
                i = (r >> 4) / each;
                h += ((r >> 4) - i * each) * 16;
            }
            h = head * p.group + (h < p.group ? h : 0);
#pragma unroll
            for (int k = 0; k < CH / 2; ++k) raw[e][k] = 0u;
            if (r < tiles * 16 && i < here) {
                const T* src = (const T*)p.Q + (size_t)(t0 + i) * p.q_stride + (size_t)h * D + CH * lane;
#pragma unroll
                for (int k = 0; k < CH / 2; ++k) raw[e][k] = *reinterpret_cast<const uint32_t*>(src + 2 * k);
            }
        }
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const int r = r0 + e * WARPS;
            if (r >= tiles * 16) break;                        // the same for the whole warp
            float x[CH], a = 0.f;
#pragma unroll
            for (int k = 0; k < CH; k += 2) {
                const float2 two = xsv_unpack2<T>(raw[e][k / 2]);
                x[k] = two.x; x[k + 1] = two.y;
                a = fmaxf(a, fmaxf(fabsf(two.x), fabsf(two.y)));
            }
            a = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(a)));
            a = fmaxf(a, 8.67361737988403547e-19f);            // 2^-60
            const float inv = __fdiv_rn(127.f, a);
            uint32_t w = 0;
#pragma unroll
            for (int k = 0; k < CH; ++k) w |= ((uint32_t)__float2int_rn(__fmul_rn(x[k], inv)) & 0xFFu) << (8 * k);
            // word n of the row (channels 4 n on) belongs to step n / 16 * 2 + n % 4 / 2, lane 4 (row % 8) + n % 16 / 4, register 2 (n % 2) + row / 8
            const int n = CH * lane / 4;
            uint8_t* const at = q8 + ((((r >> 4) * 2 * KB + n / 16 * 2 + n % 4 / 2) * 32 + 4 * (r & 7) + n % 16 / 4) * 4 + 2 * (n % 2) + (r >> 3 & 1)) * 4;
            if (CH == 4) *reinterpret_cast<uint32_t*>(at) = w;
            else reinterpret_cast<unsigned short*>(at)[lane & 1] = (unsigned short)w;
            if (lane == 0) qa[r] = a;
        }
    }
    uint32_t lead = smem_u32(keys);                            // the first block's keys
    if (CLUSTER) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");          // all blocks run: their shared memory can be written
        asm("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(lead));
    }
    __syncthreads();
    // the key of a token and page, where `is`; rows of keys have room for the pages of a whole turn
    auto store = [&](bool is, int i, int page, uint32_t key) {
        const uint32_t at = lead + 4u * (uint32_t)(i * across + page);
        if (CLUSTER) asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p st.shared::cluster.u32 [%0], %1;\n\t}" ::"r"(at), "r"(key), "r"((uint32_t)is) : "memory");
        else asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p st.shared.u32 [%0], %1;\n\t}" ::"r"(at), "r"(key), "r"((uint32_t)is) : "memory");
    };
    // ---- scores
    int id = -1;                                               // places of the next turn's pages
    for (int a = 0; a < here;) {
        const int b = run;
        for (int base = base0; base < end; base += step) {
            if (a > 0 || base > base0) fetch(base > base0 ? id : look_up(a, base));
            id = look_up(a, base + step);
            // what belongs to this lane's columns, pages 8 u + 2 j and the one after it
            unsigned long long fs[NU];
            uint32_t is[2];
#pragma unroll
            for (int u = 0; u < NU; ++u) fs[u] = f2_pack(__shfl_sync(0xFFFFFFFFu, f[u], 8 * j), __shfl_sync(0xFFFFFFFFu, f[u], 8 * j + 4));
            is[0] = __shfl_sync(0xFFFFFFFFu, there, 8 * j);
            is[1] = __shfl_sync(0xFFFFFFFFu, there, 8 * j + 4);
            // Scores of a tile's rows g and g + 8 for pages 8 u + 2 j + c: the larger of both, where they are one token's.
            auto tile = [&](int n, float (&x)[NU][2], float (&y)[NU][2]) {
                uint4 q[2 * KB];
#pragma unroll
                for (int k = 0; k < 2 * KB; ++k) q[k] = *reinterpret_cast<const uint4*>(q8 + ((n * 2 * KB + k) * 32 + lane) * 16);
                const float a0 = qa[16 * n + g], a1 = qa[16 * n + 8 + g];
                const unsigned long long down = f2_pack(-12582912.f, -12582912.f);
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    int c[4];
#pragma unroll
                    for (int k = 0; k < KB; ++k) {
                        if (k == 0) mma_s8(c, q[0].x, q[0].y, q[0].z, q[0].w, m[u][0].x, m[u][0].y, MAGIC);
                        else mma_s8(c, q[2 * k].x, q[2 * k].y, q[2 * k].z, q[2 * k].w, m[u][k].x, m[u][k].y);
                        mma_s8(c, q[2 * k + 1].x, q[2 * k + 1].y, q[2 * k + 1].z, q[2 * k + 1].w, m[u][k].z, m[u][k].w);
                    }
                    auto score = [&](int c0, int c1, float a_, float (&to)[2]) {
                        const unsigned long long dot = f2_add(f2_pack(__int_as_float(c0), __int_as_float(c1)), down);
                        f2_unpack(f2_mul(f2_mul(dot, fs[u]), f2_pack(a_, a_)), to[0], to[1]);
                    };
                    score(c[0], c[1], a0, x[u]);
                    score(c[2], c[3], a1, y[u]);
                    if (ROWS > 1) { x[u][0] = fmaxf(x[u][0], y[u][0]); x[u][1] = fmaxf(x[u][1], y[u][1]); }
                }
            };
            // The rest of the maximum over a token's rows: of the values i < N that two lanes have, the lane whose bit is clear keeps the
            // first half, the other one the second, as long as there are several; then the keys.
            auto put = [&](int i, bool live, const float (&x)[NU][2]) {
                constexpr int N0 = 2 * NU, N1 = N0 / 2, N2 = N1 / 2;      // N2: 2 or 1
                auto store_one = [&](float v, int at) {        // value `at` of the turn's: page 8 (at / 2) + 2 j + at % 2
                    store(live, i, base + 8 * (at >> 1) + 2 * j + (at & 1), ((at & 1) ? is[1] : is[0]) >> (at >> 1) & 1u ? order_of(v) : 0u);
                };
                float v[N0];
#pragma unroll
                for (int u = 0; u < NU; ++u) { v[2 * u] = x[u][0]; v[2 * u + 1] = x[u][1]; }
                const int b0 = g & 1, b1 = g >> 1 & 1, b2 = g >> 2;
                if constexpr (ROWS <= 2) {
#pragma unroll
                    for (int e = 0; e < N0; ++e) store_one(v[e], e);
                } else {
                    float v1[N1];
#pragma unroll
                    for (int e = 0; e < N1; ++e) v1[e] = fmaxf(b0 ? v[N1 + e] : v[e], __shfl_xor_sync(0xFFFFFFFFu, b0 ? v[e] : v[N1 + e], 4));
                    if constexpr (ROWS == 4) {
#pragma unroll
                        for (int e = 0; e < N1; ++e) store_one(v1[e], N1 * b0 + e);
                    } else {
                        float v2[N2];
#pragma unroll
                        for (int e = 0; e < N2; ++e) v2[e] = fmaxf(b1 ? v1[N2 + e] : v1[e], __shfl_xor_sync(0xFFFFFFFFu, b1 ? v1[e] : v1[N2 + e], 8));
                        if constexpr (ROWS == 8) {
#pragma unroll
                            for (int e = 0; e < N2; ++e) store_one(v2[e], N1 * b0 + N2 * b1 + e);
                        } else if constexpr (N2 > 1) {
                            const float one = fmaxf(b2 ? v2[1] : v2[0], __shfl_xor_sync(0xFFFFFFFFu, b2 ? v2[0] : v2[1], 16));
                            store_one(one, N1 * b0 + N2 * b1 + b2);
                        } else {                               // one left: both lanes have it
                            const float one = fmaxf(v2[0], __shfl_xor_sync(0xFFFFFFFFu, v2[0], 16));
                            if (b2 == 0) store_one(one, N1 * b0 + N2 * b1);
                        }
                    }
                }
            };
            if (ROWS < 16) {
                for (int n = a / TOKENS; n < (b + TOKENS - 1) / TOKENS; ++n) {
                    float x[NU][2], y[NU][2];
                    tile(n, x, y);
                    const int i = n * TOKENS + (ROWS == 1 ? g : g / (ROWS > 1 ? ROWS / 2 : 1));
                    put(i, i >= a && i < b, x);
                    if (ROWS == 1) put(i + 8, i + 8 >= a && i + 8 < b, y);
                }
            } else {                                           // a token's rows may be several tiles
                for (int i = a; i < b; ++i) {
                    float best[NU][2];
                    for (int n = i * each; n < (i + 1) * each; ++n) {
                        float x[NU][2], y[NU][2];
                        tile(n, x, y);
#pragma unroll
                        for (int u = 0; u < NU; ++u)
#pragma unroll
                            for (int c = 0; c < 2; ++c) best[u][c] = n == i * each ? x[u][c] : fmaxf(best[u][c], x[u][c]);
                    }
                    put(i, true, best);
                }
            }
        }
        a = b;
        if (a < here) begin_run(a);
    }
    if (CLUSTER) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank != 0) return;
    }
    __syncthreads();
    // ---- the lists
    static_assert(WARPS >= 8, "a warp for each of a block's tokens");
    if (listed < here)
        list_of<MODE == MANY ? 1 : WARPS>(p, keys + listed * across, s_seq[listed], s_mine[listed], ahead, p.out + ((size_t)(t0 + listed) * p.pool.heads + head) * p.top,
                                          s_note, MODE == MANY ? 0 : wid);
}

size_t smem_of(int tokens, int rows, int head_dim, int width) {
    const int tiles = (tokens * rows + 15) / 16;
    return (size_t)tiles * 16 * (head_dim + 4) + (size_t)tokens * key_stride(width) * 4;
}
constexpr size_t SMEM_MAX = 200 * 1024;

template <typename T, int D, int ROWS, Mode MODE> cudaError_t launch(const Select& p, long long blocks, cudaStream_t st) {
    auto kernel = page8_select_kernel<T, D, ROWS, MODE>;
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
    cfg.dynamicSmemBytes = smem_of(p.tokens, p.rows, D, p.width);
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
template <typename T, int D, int ROWS> cudaError_t launch_mode(const Select& p, long long blocks, cudaStream_t st) {
    if (p.tokens > 1) return launch<T, D, ROWS, MANY>(p, blocks, st);
    return p.cluster > 1 ? launch<T, D, ROWS, SHARED>(p, blocks, st) : launch<T, D, ROWS, ONE>(p, blocks, st);
}
template <typename T, int D> cudaError_t launch_rows(const Select& p, long long blocks, cudaStream_t st) {
    switch (p.rows) {
        case 1: return launch_mode<T, D, 1>(p, blocks, st);
        case 2: return launch_mode<T, D, 2>(p, blocks, st);
        case 4: return launch_mode<T, D, 4>(p, blocks, st);
        case 8: return launch_mode<T, D, 8>(p, blocks, st);
        default: return launch_mode<T, D, 16>(p, blocks, st);
    }
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
    p.rows = p.group > 8 ? (p.group + 15) / 16 * 16 : p.group > 4 ? 8 : p.group > 2 ? 4 : p.group;
    // Many tokens: 8 a block, a warp selects for each.  8 heads of 128 over 40 000 tokens, 8 tokens a block against one: 24 tokens of a sequence
    // 12.6 against 11.4 us, 40 tokens 13.2 against 16.8, 296 tokens 16.6 against 72.  Where they belong to as many sequences a block scores for
    // one after the other: 64 sequences 41 against 22, 128 sequences 44 against 38, 512 sequences 26 against 82.
    // Few: one a block, and 2 to 8 blocks a token while that leaves them two multiprocessors each and each has 128 pages at least (one sequence of
    // 200 000 tokens: 1 block 23.2 us, 8 blocks 13.3; 20 000: 1 block 7.1, 2 blocks 6.9; 16 sequences of 60 000: 2 blocks 13.3, 4 blocks 16.5).
    const long long units = (long long)n_tokens * pool->kv_heads;
    p.tokens = 1;
    p.cluster = 1;
    if (units >= (n_tokens >= 8LL * n_seqs ? 2LL : 8LL) * xsv_sm_count()) {
        p.tokens = 8;
        while (p.tokens > 1 && (smem_of(p.tokens, p.rows, pool->head_dim, table_width) > SMEM_MAX || p.tokens * p.rows > XSV_PAGE8_MAX_GROUP)) p.tokens /= 2;
    } else {
        while (p.cluster < 8 && units * p.cluster * 2 <= 2 * xsv_sm_count() && table_width >= 256 * p.cluster) p.cluster *= 2;
    }
    const long long blocks = ((long long)n_tokens + p.tokens - 1) / p.tokens * pool->kv_heads * p.cluster;
    if (blocks > 0x7FFFFFFFLL) return XSV_ERR_LIMIT;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (pool->dtype == XSV_F16) e = pool->head_dim == 64 ? launch_rows<__half, 64>(p, blocks, st) : launch_rows<__half, 128>(p, blocks, st);
    else e = pool->head_dim == 64 ? launch_rows<__nv_bfloat16, 64>(p, blocks, st) : launch_rows<__nv_bfloat16, 128>(p, blocks, st);
    return e == cudaSuccess ? XSV_OK : xsv_cuda_status(e);
}
