// Eq. 2 + Eq. 12: attention of one frame's queries over [dequantised cache ;
// fresh frame] on the 5th-generation tensor cores (tcgen05.mma, accumulators
// in tensor memory).
//
// Work decomposition.  A unit is (head, pair of 128-query tiles); its key/value
// sequence is cut into tiles of 128 tokens (two key quantisation groups).  The
// grid is one persistent CTA per SM; the (unit, kv-tile) steps, weighted by their
// cost, are dealt out in contiguous spans, so a unit may be shared by several
// CTAs.  A CTA that covers a whole unit writes the output rows itself; otherwise
// it writes its unnormalised accumulator with the row maxima and sums, and
// attn_combine_kernel merges the parts in a fixed order (deterministic).
//
// Inside a CTA (16 warps):
//   warps 0-3, 4-7 : softmax of query tile A / B, one query row per thread
//                    (tensor-memory lane == row), online softmax in float32 with
//                    lazy rescaling of the accumulator;
//   warps 8-13     : producers: load the packed rows of a kv tile (16-byte loads, one
//                    slab ahead), unpack the codes, dequantise in registers (Eq. 12)
//                    and write fp16 tiles to shared memory in the 128-byte-swizzled
//                    layout the MMA descriptors expect.  The operands do not exist in
//                    HBM in that form, so the tiles cannot be copied in; feeding the
//                    packed rows through a bulk-copy staging slot per warp
//                    (cp.async.bulk + mbarrier) was built and measured 12-22 % slower
//                    than the loads into registers, and is not used.  A cache kept unquantised
//                    does hold its operands in MMA form: its K and V tiles, and the frame's,
//                    are fetched by tensor-map bulk copies issued by one producer lane
//                    (cp.async.bulk.tensor, 128-byte swizzle, no multicast), fp16 or -- with
//                    bf16 operands in the MMAs -- bf16; where no tensor map can be made (an
//                    unaligned pointer) its producers stage raw slabs in shared memory by
//                    16-byte asynchronous copies and convert bf16 to fp16;
//   warps 14, 15   : one thread each issues, for query tile A / B, S = Q K^T
//                    (operands in shared memory) and O += P V (P read from tensor
//                    memory, V from shared memory).
// Stages are handed over with mbarriers; every wait is bounded and on expiry
// sets XSV_DEV_TIMEOUT in the status word, after which all waits fall through
// and the kernel runs to its end (tensor memory is always released).
//
// Operands are fp16 for both input types: bf16 inputs convert without rounding for magnitudes in [2^-14, 65504];
// smaller magnitudes are held as fp16 subnormals (absolute error at most 2^-25), larger ones saturate to +-65504
// and set XSV_DEV_RANGE in the status word.
// The channel order inside shared memory is permuted (the order in which the
// codes fall out of a packed 32-bit word); Q and fresh K rows are permuted the
// same way, and the output columns are un-permuted in the epilogue.
#include <cuda.h>

#include <algorithm>
#include <cstdlib>
#include <type_traits>

#include "tc5_ptx.cuh"
#include "xsv_kernels.h"

namespace {

constexpr int BM = 128;            // query rows per tile
constexpr int BN = 128;            // keys per kv tile
constexpr int SUB = 64;            // keys per S sub-tile: a kv tile is consumed as two halves
constexpr int NBUF = 3;            // S sub-tile buffers per query tile in tensor memory
constexpr int NSTAGE = 4;          // kv stages in shared memory
constexpr int NPROD = 6;              // producer warps
constexpr int NTHREADS = (8 + NPROD + 2) * 32;   // 8 softmax warps, the producers, one MMA issuer per query tile
constexpr uint32_t TILE_BYTES = 128u * 128u;   // 128 rows x 64 fp16
// Cost model of the work split, in ticks (fitted to per-CTA durations measured with %globaltimer): a kv step with two
// active query tiles, with one (the hand-over latencies, not the arithmetic, set the pace of a step), and the fixed
// cost of entering a unit (query tiles loaded, the first tile's rescale, the epilogue).
constexpr int COST_PAIR = 16, COST_SINGLE = 13, COST_UNIT = 72;
constexpr float SUM_LIMIT = 256.f;             // a sub-tile's row sum that reaches 2^8 (a logit 8 log2 units above the maximum in use does) triggers the careful path

// shared-memory map (from a 1024-byte aligned base)
constexpr uint32_t OFF_Q = 0;                                  // 2 tiles
constexpr uint32_t OFF_KV = 2 * TILE_BYTES;                    // NSTAGE x (K tile, V tile)
constexpr uint32_t OFF_META = OFF_KV + NSTAGE * 2 * TILE_BYTES;   // key parameters as halves: [producer warp][scale | offset][64]
constexpr uint32_t OFF_BAR = OFF_META + 3072;
constexpr uint32_t BAR_BYTES = 512;
constexpr uint32_t OFF_STAGE = OFF_BAR + BAR_BYTES;            // raw caches only: per producer warp one slab of 32 raw rows
constexpr uint32_t STAGE_BYTES = 32 * 128;
template <int BITS> constexpr uint32_t smem_bytes() {          // + alignment slack
    return OFF_STAGE + (BITS == 16 ? NPROD * STAGE_BYTES : 0u) + 1024;
}
static_assert(smem_bytes<16>() <= 227 * 1024, "shared memory");

// barrier slots (8 bytes each) inside the barrier block
enum { B_KFULL = 0, B_VFULL = NSTAGE, B_EMPTY = 2 * NSTAGE, B_SFULL = 3 * NSTAGE, B_PREADY = B_SFULL + 2 * NBUF,
       B_PVDONE = B_PREADY + 2 * NBUF, B_QFULL = B_PVDONE + 2 * NBUF, B_DRAIN = B_QFULL + 2, B_COUNT = B_DRAIN + 2 };
static_assert(B_COUNT * 8 + 16 <= BAR_BYTES, "barrier block");
// tensor-memory columns: S sub-tile buffer b of query tile x (its P, as fp16 pairs, overwrites the first half of
// the S it was computed from), then the two output accumulators
__host__ __device__ constexpr uint32_t TM_S(int x, int b) { return (uint32_t)((x * NBUF + b) * SUB); }
constexpr uint32_t TM_O0 = 2 * NBUF * SUB;
static_assert(TM_O0 + 2 * XSV_D <= 512, "tensor memory columns");
static_assert(NPROD * 2 * 64 * 2 <= 3072, "staging area of the key parameters");

struct Params {
    LayerView lv;
    const void* Q;
    const void* K;
    const void* V;
    void* out;
    float* part;        // [G][2][256][66] partial accumulators
    int* status;
    long long ticks_head, total;
    int T_c, F, H;
    int n_ct, nkv;      // cached kv tiles, all kv tiles
    int npair, n_full;  // units per head, of which with both query tiles active
    int G;              // CTAs
};

constexpr int PART_STRIDE = 256 * 66;   // floats per (CTA, slot)

// Several independent streams (caches) in one launch: stream s owns the CTAs [cta_base[s], cta_base[s + 1]) and the
// units [unit_base[s], unit_base[s + 1]) of the merge grid; each stream's Params carries its own CTA count G, its
// slice of the workspace and its own status word, so inside a CTA everything is as for a launch of that stream alone.
// Tensor maps of one stream for the copy-engine feed of an unquantised fp16 cache: cached keys, cached values, the
// frame's keys, the frame's values, each a [heads][rows][64] tensor read in boxes of 128 rows.
struct alignas(64) StreamMaps { CUtensorMap m[4]; };

struct BatchParams {
    int n;
    int use_tma;         // every stream's K / V tiles are fetched by tensor-map bulk copies (bits == 16)
    int cta_base[XSV_MAX_BATCH + 1];
    int unit_base[XSV_MAX_BATCH + 1];
    Params p[XSV_MAX_BATCH];
    StreamMaps tm[XSV_MAX_BATCH];
};

// ------------------------------------------------------------------ work split
struct Span { int kv0, kv1; };

// A unit's ticks: COST_UNIT, then its kv steps.  Inside a head the units with two active query tiles come first.
__host__ __device__ inline long long unit_len(const Params& p, bool pair) {
    return (long long)(pair ? COST_PAIR : COST_SINGLE) * p.nkv + COST_UNIT;
}
__host__ __device__ inline void unit_base_cost(const Params& p, int u, long long& base, int& cost) {
    const int h = u / p.npair, mp = u - h * p.npair;
    cost = mp < p.n_full ? COST_PAIR : COST_SINGLE;
    base = h * p.ticks_head + (long long)(mp < p.n_full ? mp : p.n_full) * unit_len(p, true) +
           (long long)(mp > p.n_full ? mp - p.n_full : 0) * unit_len(p, false);
}
__host__ __device__ inline int unit_of_tick(const Params& p, long long t) {
    const long long h = t / p.ticks_head, r = t - h * p.ticks_head;
    long long mp = r / unit_len(p, true);
    if (mp > p.n_full) mp = p.n_full + (r - p.n_full * unit_len(p, true)) / unit_len(p, false);
    if (mp >= p.npair) mp = p.npair - 1;
    return (int)(h * p.npair + mp);
}
__host__ __device__ inline long long cta_tick(const Params& p, int b) { return p.total * b / p.G; }
// kv tiles of unit u that CTA b processes: those whose first tick lies in the CTA's span
__host__ __device__ inline Span cta_span(const Params& p, int b, int u) {
    long long base;
    int cost;
    unit_base_cost(p, u, base, cost);
    const long long t0 = cta_tick(p, b) - base - COST_UNIT, t1 = cta_tick(p, b + 1) - base - COST_UNIT;   // kv step j starts at tick j * cost
    long long a = t0 <= 0 ? 0 : (t0 + cost - 1) / cost, e = t1 <= 0 ? 0 : (t1 + cost - 1) / cost;
    if (a > p.nkv) a = p.nkv;
    if (e > p.nkv) e = p.nkv;
    return Span{(int)a, (int)e};
}

// kind::f16, fp16 x fp16 -> fp32, M = 128
constexpr uint32_t IDESC_QK = (1u << 4) | ((uint32_t)(SUB >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);                 // A, B K-major, N = 64
constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 16) | ((uint32_t)(XSV_D >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);   // B MN-major, N = 64

// Channel held at shared-memory position p: the codes of one packed 32-bit word
// (W channels) come out as pairs (i, i + W/2).  W == 2 is the identity.
template <int W> __host__ __device__ constexpr int perm(int p) { return W * (p / W) + (p % W) / 2 + (W / 2) * (p % 2); }
template <int W> __host__ __device__ constexpr int inv_perm(int c) {
    return W * (c / W) + ((c % W) < W / 2 ? 2 * (c % W) : 2 * ((c % W) - W / 2) + 1);
}

// Nonzero iff one of the two bf16 halves of w has magnitude 2^16 or more (exponent field >= 143; Inf and NaN too),
// i.e. converts to fp16 by saturation.  Carry-free: each masked half is at most 0x7F80.
template <typename T> __device__ __forceinline__ uint32_t beyond_h2(uint32_t w);
template <> __device__ __forceinline__ uint32_t beyond_h2<__half>(uint32_t) { return 0u; }
template <> __device__ __forceinline__ uint32_t beyond_h2<__nv_bfloat16>(uint32_t w) {
    return ((w & 0x7F807F80u) + 0x38803880u) & 0x80008000u;
}

// One row of 64 16-bit values (global) -> fp16, permuted, one swizzled 128-byte
// row of a shared-memory tile.  grow == nullptr writes zeros.  Returns nonzero if a
// value lay beyond the fp16 range (bf16 inputs only).
// 16 channels (8 input words: block blk of a row) -> fp16, permuted, two 16-byte chunks of the tile's row.  Returns
// nonzero if a value lay beyond the fp16 range (bf16 inputs only).
template <typename T, int W>
__device__ __forceinline__ uint32_t block16_to_tile(const uint32_t (&in)[8], uint8_t* tile, int row, int blk) {
    uint32_t beyond = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) beyond |= beyond_h2<T>(in[i]);
    uint32_t o[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const int a = perm<W>(2 * q), b = perm<W>(2 * q + 1);   // local channels (W <= 16 keeps them in this block)
        const uint32_t wa = in[a >> 1], wb = in[b >> 1];
        const uint32_t lo = (a & 1) ? (wa >> 16) : (wa & 0xFFFFu);
        const uint32_t hi = (b & 1) ? (wb & 0xFFFF0000u) : (wb << 16);
        o[q] = to_h2<T>(lo | hi);
    }
    *reinterpret_cast<uint4*>(tile + swz(row, 2 * blk)) = make_uint4(o[0], o[1], o[2], o[3]);
    *reinterpret_cast<uint4*>(tile + swz(row, 2 * blk + 1)) = make_uint4(o[4], o[5], o[6], o[7]);
    return beyond;
}
template <typename T, int W>
__device__ __forceinline__ uint32_t row16_to_tile(const T* grow, uint8_t* tile, int row) {
    uint32_t beyond = 0u;
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {   // 16 channels = 8 input words = two 16-byte chunks
        uint32_t in[8];
        if (grow) {
            const uint4 a = reinterpret_cast<const uint4*>(grow)[2 * blk], b = reinterpret_cast<const uint4*>(grow)[2 * blk + 1];
            in[0] = a.x; in[1] = a.y; in[2] = a.z; in[3] = a.w; in[4] = b.x; in[5] = b.y; in[6] = b.z; in[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) in[i] = 0u;
        }
        beyond |= block16_to_tile<T, W>(in, tile, row, blk);
    }
    return beyond;
}
// The same for a row already in registers (its eight 16-byte pieces in order)
template <typename T, int W>
__device__ __forceinline__ uint32_t row_regs_to_tile(const uint4 (&rw)[8], uint8_t* tile, int row) {
    uint32_t beyond = 0u;
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {
        const uint32_t in[8] = {rw[2 * blk].x, rw[2 * blk].y, rw[2 * blk].z, rw[2 * blk].w,
                                rw[2 * blk + 1].x, rw[2 * blk + 1].y, rw[2 * blk + 1].z, rw[2 * blk + 1].w};
        beyond |= block16_to_tile<T, W>(in, tile, row, blk);
    }
    return beyond;
}

// In-register unpack.  The codes of one packed 32-bit word come out as pairs
// (i, i + W/2), W = 32 / BITS codes per word.  A pair is masked (after at most
// one shift per word half) into the mantissas of two fp16 whose exponent makes the
// unit in the last place at the code's position worth 1: with the code at mantissa
// bit TB the fp16 reads OFF + code, OFF = 1024 >> TB, exactly.
template <int BITS> __host__ __device__ constexpr int unpack_shift(int i) {   // right shift applied to the word
    return BITS == 4 ? (i < 2 ? 0 : 8) : BITS == 2 ? (i < 5 ? 0 : 10) : (i == 0 ? 0 : 8);
}
template <int BITS> __host__ __device__ constexpr int unpack_tb(int i) {      // mantissa bit of the code afterwards
    return BITS == 4 ? 4 * (i & 1) : BITS == 2 ? (i < 5 ? 2 * i : 2 * (i - 5)) : 0;
}

// half2 (OFF_i + code_i, OFF_i + code_{i + W/2}) of packed word w; i is a compile-time
// constant after unrolling
template <int BITS>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int i) {
    const int tb = unpack_tb<BITS>(i);
    const uint32_t m1 = ((1u << BITS) - 1u) << tb;
    const uint32_t magic = (uint32_t)(25 - tb) << 10;
    return ((w >> unpack_shift<BITS>(i)) & (m1 | (m1 << 16))) | (magic | (magic << 16));
}
// Eq. 12 on a pair of codes: ((OFF + code) - OFF) * s + z with s the scale and z the offset of the group, both
// rounded to fp16.  The subtraction is exact (OFF is the power of two that code_pair put into the exponent), so the
// error is that of rounding s, z and the result: about one unit in the last place of the values themselves.
template <int BITS>
__device__ __forceinline__ uint32_t dq_pair(uint32_t w, int i, uint32_t s2, uint32_t z2) {
    const uint32_t off = (uint32_t)(25 - unpack_tb<BITS>(i)) << 10;          // fp16 OFF
    return hfma2_u(hsub2_u(code_pair<BITS>(w, i), off | (off << 16)), s2, z2);
}

__device__ __forceinline__ uint16_t f2h_sat(float x) {
    uint16_t h;
    asm("cvt.rn.satfinite.f16.f32 %0, %1;" : "=h"(h) : "f"(x));
    return h;
}

// 32 logits of one row -> 32 probabilities 2^(s * sc - m) packed as fp16 pairs; their sum is added to the two
// lanes of ls2.  Whole sub-tiles only.  The scaling and the sum run as packed float32 pairs (half the issue slots).
template <bool BF>
__device__ __forceinline__ void softmax32_fast(const uint32_t (&v)[32], unsigned long long sc2, unsigned long long nm2,
                                               unsigned long long& ls2, uint32_t (&pk)[16]) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float x0, x1;
        f2_unpack(f2_fma(f2_pack(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), sc2, nm2), x0, x1);
        const float p0 = ex2(x0), p1 = ex2(x1);
        ls2 = f2_add(ls2, f2_pack(p0, p1));
        pk[i >> 1] = pack_p<BF>(p0, p1);
    }
}
// The same with a mask: columns at or beyond `valid` (a ragged last tile) give probability 0.
template <bool MASK, bool BF>
__device__ __forceinline__ void softmax32(const uint32_t (&v)[32], float sc, float nm, int valid, float& ls, uint32_t (&pk)[16]) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float p0 = ex2(fmaf(__uint_as_float(v[i]), sc, nm)), p1 = ex2(fmaf(__uint_as_float(v[i + 1]), sc, nm));
        if (MASK) {
            if (i >= valid) p0 = 0.f;
            if (i + 1 >= valid) p1 = 0.f;
        }
        ls += p0 + p1;
        pk[i >> 1] = pack_p<BF>(p0, p1);
    }
}
// running maximum of 32 raw logits (the first `valid` of them)
template <bool MASK>
__device__ __forceinline__ float max32(const uint32_t (&v)[32], int valid, float mx) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float s0 = __uint_as_float(v[i]), s1 = __uint_as_float(v[i + 1]);
        if (MASK) {
            if (i >= valid) s0 = -INFINITY;
            if (i + 1 >= valid) s1 = -INFINITY;
        }
        mx = fmax3(mx, s0, s1);
    }
    return mx;
}

// What every role needs to know about its CTA.
struct Cta {
    uint8_t* smem;            // 1024-byte aligned base of the dynamic shared memory
    uint32_t smem_base;       // the same as a shared-window address
    uint32_t bar_base;        // first mbarrier
    uint32_t tmem_base;       // first allocated tensor-memory column
    volatile int* abort_flag;
    int b, u_first, u_last;   // CTA index, first and last unit of its span
};

// Walks the (unit, kv tile) steps of a CTA's span in order.
struct TileIter {
    int u, kv, kv1, h;
    bool valid;
};
__device__ __forceinline__ void tile_iter_settle(const Params& p, int b, int u_last, TileIter& t) {
    while (t.u <= u_last) {            // skip units in which this CTA has no step
        const Span sp = cta_span(p, b, t.u);
        if (sp.kv0 < sp.kv1) {
            t.kv = sp.kv0;
            t.kv1 = sp.kv1;
            t.h = t.u / p.npair;
            t.valid = true;
            return;
        }
        ++t.u;
    }
    t.valid = false;
}
__device__ __forceinline__ void tile_iter_next(const Params& p, int b, int u_last, TileIter& t) {
    if (++t.kv < t.kv1) return;
    ++t.u;
    tile_iter_settle(p, b, u_last, t);
}

// What a producer lane fetches from HBM for its row of one slab of a quantised
// kv tile: the packed row, and either the row's value parameters or (key slab)
// the key parameters of two channels, which the warp shares through shared memory.
template <int NW>
struct SlabRegs {
    uint32_t w[NW];
    float s0, s1, z0, z1;
    bool valid;
};

// Producer warps.  A kv tile is eight slabs: 32 rows of keys (slabs 0-3) or of
// values (slabs 4-7); slabs are dealt to the NPROD producer warps round-robin, one
// row per lane.  The global loads of a warp's next slab are issued before its
// current slab is unpacked, so that their latency is covered.  Kept out of line
// so that its register allocation does not weigh on the softmax path.
template <typename T, int BITS>
__device__ __noinline__ void producer_loop(const Params& p, const Cta c) {
    constexpr int W = BITS == 16 ? 2 : 32 / BITS;
    constexpr int UB = BITS == 16 ? 4 : BITS;        // the unpack code must compile for raw caches too
    constexpr int ROWB = XSV_D * BITS / 8;
    constexpr int NW = BITS == 16 ? 1 : ROWB / 4;    // packed words per row
    constexpr int SPW = (32 / UB) / 2;               // half2 slots per word
    uint8_t* const smem = c.smem;
    volatile int* const abort_flag = c.abort_flag;
    const int b = c.b, u_last = c.u_last;
    auto BAR = [&](int i) { return c.bar_base + 8u * (uint32_t)i; };
    const int lane = threadIdx.x & 31, pw = (threadIdx.x >> 5) - 8;   // producer warp 0 .. NPROD-1
    const T* Kg = reinterpret_cast<const T*>(p.K);
    const T* Vg = reinterpret_cast<const T*>(p.V);
    const int F = p.F, n_ct = p.n_ct, T_c = p.T_c;
    int* const status = p.status;
    // Quantised caches read the view from the kernel's parameter space where they use it: a copy in registers makes
    // the 8-bit unpacking spill its prefetched words, and a spilled prefetch waits for the load it was meant to hide
    // (8-bit: 0.36 -> 0.24 ms per layer-step).  The raw path has the registers and is faster with the copy.
    typename std::conditional<BITS == 16, const LayerView, const LayerView&>::type lv = p.lv;
    uint16_t* const mS = reinterpret_cast<uint16_t*>(smem + OFF_META) + pw * 128;   // this warp's [scale | offset][64] as fp16
    uint16_t* const mB = mS + 64;

    // slab g of the CTA: tile g / 8, slab g % 8; this warp owns g = pw, pw + NPROD, ...
    auto fetch = [&](const TileIter& ti, int sl, SlabRegs<NW>& r) {
        if (BITS == 16 || !ti.valid || ti.kv >= n_ct) return;
        const int tok = ti.kv * BN + (sl & 3) * 32 + lane;
        r.valid = tok < T_c;
        const size_t row = (size_t)ti.h * lv.cap + (r.valid ? tok : 0);
        const uint4* src = reinterpret_cast<const uint4*>((sl < 4 ? lv.kcodes : lv.vcodes) + row * ROWB);
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) {
            const uint4 a = src[i];
            r.w[4 * i] = a.x; r.w[4 * i + 1] = a.y; r.w[4 * i + 2] = a.z; r.w[4 * i + 3] = a.w;
        }
        if (sl < 4) {                       // key parameters of the channels at positions lane and lane + 32
            const int grp = ti.kv * 2 + ((sl & 3) >> 1);
            r.s0 = r.s1 = 0.f;
            r.z0 = r.z1 = 0.f;
            if (grp * XSV_G < T_c) {
                const size_t m = ((size_t)ti.h * lv.capg + grp) * 64;
                r.s0 = lv.kscale[m + perm<W>(lane)];
                r.z0 = lv.kzero[m + perm<W>(lane)];
                r.s1 = lv.kscale[m + perm<W>(lane + 32)];
                r.z1 = lv.kzero[m + perm<W>(lane + 32)];
            }
        } else {
            r.s0 = lv.vscale[row];
            r.z0 = lv.vzero[row];
        }
    };

    // A cache kept unquantised (BITS == 16): the slab's 32 raw rows (4 KB, contiguous in memory) are copied
    // asynchronously into this warp's staging slot one slab ahead -- lane l moves bytes [512 k + 16 l, + 16), k < 8, so a
    // copy instruction covers 512 consecutive bytes -- with the 16-byte piece p of row r at position p ^ (r & 7) of the
    // row, so that the copies in (8 lanes per row) and the reads out (one row per lane) are free of bank conflicts.
    // Rows past the end are filled with zeros (source size 0).
    uint8_t* const slot = smem + OFF_STAGE + (uint32_t)pw * STAGE_BYTES;
    auto stage = [&](const TileIter& ti, int sl) {
        if (ti.valid) {
            const bool cached = ti.kv < n_ct;
            const int t0 = (cached ? ti.kv : ti.kv - n_ct) * BN + (sl & 3) * 32, lim = cached ? T_c : F;
            const uint8_t* base = cached ? (sl < 4 ? lv.kcodes : lv.vcodes) + (size_t)ti.h * lv.cap * (XSV_D * 2)
                                         : reinterpret_cast<const uint8_t*>(sl < 4 ? Kg : Vg) + (size_t)ti.h * F * (XSV_D * 2);
            const uint32_t dst0 = smem_u32(slot);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = 4 * k + (lane >> 3), pc = lane & 7;
                const bool ok = t0 + r < lim;
                cp_async16(dst0 + swz(r, pc), base + (ok ? (size_t)(t0 + r) * (XSV_D * 2) + 16 * pc : 0), ok ? 16u : 0u);
            }
        }
        cp_async_commit();
    };

    uint32_t beyond = 0u;                           // a raw 16-bit input outside the fp16 range was seen
    TileIter cur{c.u_first, 0, 0, 0, false}, nxt;
    tile_iter_settle(p, b, u_last, cur);
    uint32_t it = 0;                                // kv tile of `cur`
    uint32_t g = (uint32_t)pw;                      // this warp's current slab
    auto seek = [&](TileIter& ti, uint32_t& ti_it, uint32_t tile) {   // advance an iterator to kv tile `tile`
        while (ti.valid && ti_it < tile) {
            tile_iter_next(p, b, u_last, ti);
            ++ti_it;
        }
    };
    seek(cur, it, g >> 3);
    SlabRegs<NW> rc{}, rn{};
    if (BITS == 16) stage(cur, (int)(g & 7u));
    else fetch(cur, (int)(g & 7u), rc);
    while (cur.valid) {
        const int sl = (int)(g & 7u);
        // the next slab of this warp: start its loads now
        const uint32_t gn = g + NPROD;
        nxt = cur;
        uint32_t itn = it;
        seek(nxt, itn, gn >> 3);
        uint4 rw[8];
        if (BITS == 16) {
            // this slab's row out of the staging slot, then the slot is free for the next slab's copies
            cp_async_wait_all();
            __syncwarp();
#pragma unroll
            for (int pc = 0; pc < 8; ++pc) rw[pc] = *reinterpret_cast<const uint4*>(slot + swz(lane, pc));
            __syncwarp();
            stage(nxt, (int)(gn & 7u));
        } else {
            fetch(nxt, (int)(gn & 7u), rn);
        }

        const uint32_t st = it % NSTAGE;
        uint8_t* tile = smem + OFF_KV + st * 2 * TILE_BYTES + (sl < 4 ? 0u : TILE_BYTES);
        const int row = (sl & 3) * 32 + lane;
        if (it >= NSTAGE) mbar_wait(BAR(B_EMPTY + st), ((it / NSTAGE) - 1u) & 1u, abort_flag, status, XSV_DEV_SITE_STAGE);
        const bool cached = cur.kv < n_ct;
        if (BITS < 16 && cached) {
            if (sl < 4) {
                // keys: stage the group's per-channel parameters (fp16, position order), then unpack the row
                __syncwarp();                      // the previous slab's reads of the staging area are over
                mS[lane] = f2h_sat(rc.s0); mB[lane] = f2h_sat(rc.z0);
                mS[lane + 32] = f2h_sat(rc.s1); mB[lane + 32] = f2h_sat(rc.z1);
                __syncwarp();
                const uint4* s4p = reinterpret_cast<const uint4*>(mS);
                const uint4* b4p = reinterpret_cast<const uint4*>(mB);
#pragma unroll
                for (int ck = 0; ck < 8; ++ck) {   // 16-byte chunk = half2 slots 4ck .. 4ck+3
                    const uint4 s4 = s4p[ck], b4 = b4p[ck];
                    const uint32_t sv[4] = {s4.x, s4.y, s4.z, s4.w}, bv[4] = {b4.x, b4.y, b4.z, b4.w};
                    uint32_t o[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int slot = 4 * ck + q;
                        o[q] = dq_pair<UB>(rc.w[(slot / SPW) % NW], slot % SPW, sv[q], bv[q]);
                    }
                    *reinterpret_cast<uint4*>(tile + swz(row, ck)) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            } else {
                // values: the row's own scale and offset
                const uint32_t sh = f2h_sat(rc.s0), zh = f2h_sat(rc.z0);
                const uint32_t s2 = sh | (sh << 16), z2 = zh | (zh << 16);
#pragma unroll
                for (int ck = 0; ck < 8; ++ck) {
                    uint32_t o[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int slot = 4 * ck + q;
                        o[q] = dq_pair<UB>(rc.w[(slot / SPW) % NW], slot % SPW, s2, z2);
                    }
                    *reinterpret_cast<uint4*>(tile + swz(row, ck)) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
            if (!rc.valid) {                       // rows past the end of the cache (last tile only) read as zero
#pragma unroll
                for (int ck = 0; ck < 8; ++ck) *reinterpret_cast<uint4*>(tile + swz(row, ck)) = make_uint4(0u, 0u, 0u, 0u);
            }
        } else if (BITS == 16) {
            beyond |= row_regs_to_tile<T, W>(rw, tile, row);     // rows past the end were staged as zeros
        } else {
            // raw 16-bit rows of the fresh frame
            const T* src = nullptr;
            if (cached) {
                const int tok = cur.kv * BN + row;
                if (tok < T_c)
                    src = reinterpret_cast<const T*>(sl < 4 ? lv.kcodes : lv.vcodes) + ((size_t)cur.h * lv.cap + tok) * XSV_D;
            } else {
                const int tok = (cur.kv - n_ct) * BN + row;
                if (tok < F) src = (sl < 4 ? Kg : Vg) + ((size_t)cur.h * F + tok) * XSV_D;
            }
            beyond |= row16_to_tile<T, W>(src, tile, row);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR((sl < 4 ? B_KFULL : B_VFULL) + st));
        rc = rn;
        cur = nxt;
        it = itn;
        g = gn;
    }
    if (beyond) atomicOr(status, XSV_DEV_RANGE);
}

// Copy-engine feed for a cache kept unquantised with fp16 inputs: the operands exist in HBM in the form the MMA reads
// (rows of 64 fp16, no conversion, identity channel order), so one lane asks the copy engine for whole K and V tiles
// -- boxes of 128 rows x 128 bytes of a [heads][rows][64] tensor map, written in the 128-byte-swizzled layout of the MMA
// descriptors; rows past the end of the cache or of the frame arrive as zeros -- and the other producer lanes have
// nothing to do.  The byte counts complete the stage's KFULL / VFULL barriers (one announcing arrival each).
__device__ __noinline__ void producer_tma_loop(const Params& p, const Cta c, const StreamMaps& maps) {
    if (threadIdx.x != 8 * 32) return;              // lane 0 of the first producer warp
    auto BAR = [&](int i) { return c.bar_base + 8u * (uint32_t)i; };
    volatile int* const abort_flag = c.abort_flag;
    const int n_ct = p.n_ct;
    TileIter cur{c.u_first, 0, 0, 0, false};
    tile_iter_settle(p, c.b, c.u_last, cur);
    uint32_t it = 0;
    for (; cur.valid; ++it, tile_iter_next(p, c.b, c.u_last, cur)) {
        const uint32_t st = it % NSTAGE;
        if (it >= NSTAGE) mbar_wait(BAR(B_EMPTY + st), ((it / NSTAGE) - 1u) & 1u, abort_flag, p.status, XSV_DEV_SITE_STAGE);
        if (*abort_flag) break;                       // nothing is issued any more
        const bool cached = cur.kv < n_ct;
        const int row0 = (cached ? cur.kv : cur.kv - n_ct) * BN;
        const uint32_t kdst = c.smem_base + OFF_KV + st * 2 * TILE_BYTES, vdst = kdst + TILE_BYTES;
        mbar_expect_tx(BAR(B_KFULL + (int)st), TILE_BYTES);
        tma_load_3d(kdst, &maps.m[cached ? 0 : 2], BAR(B_KFULL + (int)st), 0, row0, cur.h);
        mbar_expect_tx(BAR(B_VFULL + (int)st), TILE_BYTES);
        tma_load_3d(vdst, &maps.m[cached ? 1 : 3], BAR(B_VFULL + (int)st), 0, row0, cur.h);
    }
    // the copies that may still be in flight land before the block can end, also where no one waits for them any more
    for (uint32_t i = it > NSTAGE ? it - NSTAGE : 0; i < it; ++i) {
        mbar_wait_bounded(BAR(B_KFULL + (int)(i % NSTAGE)), (i / NSTAGE) & 1u);
        mbar_wait_bounded(BAR(B_VFULL + (int)(i % NSTAGE)), (i / NSTAGE) & 1u);
    }
}

// One row of 64 16-bit values copied as it is (identity channel order) into a swizzled row of a tile; zeros for null.
__device__ __forceinline__ void row16_raw_to_tile(const void* grow, uint8_t* tile, int row) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *reinterpret_cast<uint4*>(tile + swz(row, i)) = grow ? reinterpret_cast<const uint4*>(grow)[i] : make_uint4(0u, 0u, 0u, 0u);
}

// Softmax warpgroups (warps 0-3: query tile A, warps 4-7: tile B) and the epilogue.  BF: the MMA operands are bf16
// (an unquantised bf16 cache fed by the copy engine): the queries go in unconverted and the probabilities are packed
// as bf16 pairs.
template <typename T, int BITS, bool BF>
__device__ __noinline__ void softmax_loop(const Params& p, const Cta cta) {
    constexpr int W = BITS == 16 ? 2 : 32 / BITS;
    uint8_t* const smem = cta.smem;
    const uint32_t tmem_base = cta.tmem_base;
    volatile int* const abort_flag = cta.abort_flag;
    const int b = cta.b, u_first = cta.u_first, u_last = cta.u_last;
    auto BAR = [&](int i) { return cta.bar_base + 8u * (uint32_t)i; };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const T* Qg = reinterpret_cast<const T*>(p.Q);
    T* Og = reinterpret_cast<T*>(p.out);
    const int F = p.F, nkv = p.nkv, n_ct = p.n_ct, T_c = p.T_c;
    int* const status = p.status;
    {
        // =============================================================== softmax + epilogue
        const int X = warp >> 2;                       // query tile of this warpgroup
        const int row = tid & 127;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem_base + lane_base + TM_S(X, 0);
        const uint32_t tO = tmem_base + lane_base + TM_O0 + (uint32_t)(X * XSV_D);
        uint8_t* sQ = smem + OFF_Q + X * TILE_BYTES;
        const float SC = 0.125f * 1.4426950408889634f;   // 1/sqrt(64) * log2(e)
        uint32_t cX = 0;                               // sub-tiles of this query tile so far (all units of the CTA)
        // Completion of the P V of sub-tile j (and of every MMA issued before it).  One barrier per S buffer: a parity
        // wait is only meaningful while the barrier is at most one phase ahead, and the barrier of buffer j % NBUF
        // cannot complete again before this warp has handed over the P of sub-tile j + NBUF; its previous phase
        // (sub-tile j - NBUF) is known complete once S of sub-tile j' >= j has been received.
        auto wait_pv = [&](uint32_t j) {
            mbar_wait(BAR(B_PVDONE + X * NBUF + (int)(j % NBUF)), (j / NBUF) & 1u, abort_flag, status, XSV_DEV_SITE_PV);
        };
        for (int u = u_first; u <= u_last; ++u) {
            const Span sp = cta_span(p, b, u);
            if (sp.kv0 >= sp.kv1) continue;
            const int h = u / p.npair, mp = u - h * p.npair;
            const int q0 = mp * 2 * BM + X * BM;
            if (q0 >= F) continue;                     // second tile of the last pair may be empty
            const int grow = q0 + row;
            // ---- this unit's queries -> shared memory (all MMAs reading the previous unit's tile are complete:
            //      the last S of that unit has been received)
            if (BF) row16_raw_to_tile(grow < F ? Qg + ((size_t)h * F + grow) * XSV_D : nullptr, sQ, row);
            else if (row16_to_tile<T, W>(grow < F ? Qg + ((size_t)h * F + grow) * XSV_D : nullptr, sQ, row)) atomicOr(status, XSV_DEV_RANGE);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(B_QFULL + X));

            // Online softmax over sub-tiles of 64 keys.  S arrives in one of NBUF buffers (the QK^T of the next
            // sub-tiles are already in flight or done while this one is worked on); the probabilities, as fp16
            // pairs, overwrite the first half of the buffer they were computed from.
            //
            // The row maximum in use, m_used, is updated lazily.  The usual path does not look for the maximum at
            // all: it exponentiates with m_used and watches the row sum of the sub-tile.  A logit more than
            // 8 (log2 units) above m_used makes that sum reach SUM_LIMIT = 2^8; then (and on
            // a span's first sub-tile, and on ragged ones) the careful path below finds the true maximum, rescales
            // the accumulator and the running sum if it lies above m_used, and redoes the sub-tile from the
            // logits, which are still in registers.  A sum that large without such a logit only costs the redo.
            float m_used = -INFINITY, l = 0.f;
            bool first = true;
            for (int kv = sp.kv0; kv < sp.kv1; ++kv) {
                const int cnt = kv < n_ct ? min(BN, T_c - kv * BN) : min(BN, F - (kv - n_ct) * BN);
                for (int sub = 0; sub * SUB < cnt; ++sub) {
                    const int valid = cnt - sub * SUB;             // >= SUB: a whole sub-tile
                    const uint32_t buf = cX % NBUF;
                    const uint32_t tSb = tS + buf * SUB;
                    mbar_wait(BAR(B_SFULL + X * NBUF + (int)buf), (cX / NBUF) & 1u, abort_flag, status, XSV_DEV_SITE_S);
                    tc_fence_after();
                    uint32_t va[32], vb[32], pk[16];
                    tmem_ld32(tSb, va);
                    tmem_ld32(tSb + 32u, vb);
                    tc_wait_ld();
                    float ls = 0.f;
                    bool careful = first || valid < SUB;           // uniform
                    if (!careful) {
                        const unsigned long long sc2 = f2_pack(SC, SC), nm2 = f2_pack(-m_used, -m_used);
                        unsigned long long ls2 = f2_pack(0.f, 0.f);
                        softmax32_fast<BF>(va, sc2, nm2, ls2, pk);
                        tmem_st16(tSb, pk);
                        softmax32_fast<BF>(vb, sc2, nm2, ls2, pk);
                        tmem_st16(tSb + 16u, pk);
                        float l0, l1;
                        f2_unpack(ls2, l0, l1);
                        ls = l0 + l1;
                        careful = __any_sync(0xFFFFFFFFu, !(ls < SUM_LIMIT));
                    }
                    if (careful) {
                        float mx;
                        if (valid >= SUB) mx = max32<false>(vb, 32, max32<false>(va, 32, -INFINITY));
                        else mx = max32<true>(vb, valid - 32, max32<true>(va, valid, -INFINITY));
                        const float m_new = mx * SC;
                        const bool need = m_new > m_used;
                        if (__any_sync(0xFFFFFFFFu, need)) {
                            // rescale the accumulator and the row sum (the previous sub-tile's P V must have completed)
                            if (!first) {
                                wait_pv(cX - 1u);
                                tc_fence_after();
                            }
                            const float alpha = need ? ex2(m_used - m_new) : 1.f;
                            if (need) m_used = m_new;
                            l *= alpha;
                            if (!first) {
#pragma unroll 1
                                for (int c = 0; c < 4; ++c) {
                                    uint32_t o[16];
                                    tmem_ld16(tO + 16u * c, o);
                                    tc_wait_ld();
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                    tmem_st16(tO + 16u * c, o);
                                }
                            }
                        }
                        const float nm = -m_used;
                        ls = 0.f;
                        if (valid >= SUB) {
                            softmax32<false, BF>(va, SC, nm, 32, ls, pk);
                            tmem_st16(tSb, pk);
                            softmax32<false, BF>(vb, SC, nm, 32, ls, pk);
                            tmem_st16(tSb + 16u, pk);
                        } else {
                            softmax32<true, BF>(va, SC, nm, valid, ls, pk);
                            tmem_st16(tSb, pk);
                            softmax32<true, BF>(vb, SC, nm, valid - 32, ls, pk);
                            tmem_st16(tSb + 16u, pk);
                        }
                    }
                    l += ls;
                    tc_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(BAR(B_PREADY + X * NBUF + (int)buf));
                    ++cX;
                    first = false;
                }
            }
            // ---- epilogue of the span
            wait_pv(cX - 1u);
            tc_fence_after();
            const bool full = sp.kv0 == 0 && sp.kv1 == nkv;
            const float inv = 1.f / l;
            float* part = p.part + ((size_t)b * 2 + (sp.kv0 > 0 ? 0 : 1)) * PART_STRIDE;
#pragma unroll
            for (int c = 0; c < 4; ++c) {          // 16 positions = 16 channels (the permutation stays inside)
                uint32_t o[16];
                tmem_ld16(tO + 16u * c, o);
                tc_wait_ld();
                if (full) {
                    if (grow < F) {
                        uint32_t w[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) {    // channels 16c + 2q, 16c + 2q + 1
                            const float a = __uint_as_float(o[inv_perm<W>(16 * c + 2 * q) - 16 * c]) * inv;
                            const float bb = __uint_as_float(o[inv_perm<W>(16 * c + 2 * q + 1) - 16 * c]) * inv;
                            w[q] = xsv_pack2<T>(a, bb);
                        }
                        uint4* dst = reinterpret_cast<uint4*>(Og + ((size_t)h * F + grow) * XSV_D + 16 * c);
                        dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                        dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                } else {
                    float4* dst = reinterpret_cast<float4*>(part + (size_t)(X * BM + row) * 64 + 16 * c);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        dst[q] = make_float4(__uint_as_float(o[inv_perm<W>(16 * c + 4 * q) - 16 * c]),
                                             __uint_as_float(o[inv_perm<W>(16 * c + 4 * q + 1) - 16 * c]),
                                             __uint_as_float(o[inv_perm<W>(16 * c + 4 * q + 2) - 16 * c]),
                                             __uint_as_float(o[inv_perm<W>(16 * c + 4 * q + 3) - 16 * c]));
                }
            }
            if (!full) {
                float2* ml = reinterpret_cast<float2*>(part + 256 * 64);
                ml[X * BM + row] = make_float2(m_used, l);
            }
            tc_fence_before();   // the accumulator has been read: orders these loads before this thread's next arrive
        }
    }
}

// MMA issuers: one warp per query tile, each running converged; the tensor-core instructions and their commits
// are issued by its elected lane.
//
// Tile x consumes the span's kv tiles as sub-tiles of 64 keys: S_j = Q K_j^T into buffer j % NBUF, then (once the
// softmax warps have turned S_j into P_j in place) O += P_j V_j.  The tensor pipe executes the MMAs of one thread
// in issue order, so QK(j + NBUF) is issued right behind PV(j) into the buffer that PV(j) reads: no barrier is
// needed for the reuse, and NBUF QK^T run ahead of the softmax.
//
// The order of issue is fixed -- PV(j), QK(j + NBUF), j = 0, 1, ... -- and every counter is a loop variable that
// depends on the kernel parameters and the block index only, never on the outcome of a barrier test; that keeps
// the operands of the tcgen05 instructions (descriptors, tensor-memory addresses, barrier addresses) uniform.
// What sets the pace of this loop is the chain of waits, fences and elections around each group of four MMAs,
// not the MMAs themselves (which execute in 35-52 clocks each), hence one such loop per query tile.
constexpr uint32_t IDESC_BF16 = (1u << 7) | (1u << 10);     // A and B are bf16 instead of fp16
__device__ __noinline__ void mma_loop(const Params& p, const Cta c, const int x, const uint32_t fmt) {
    const uint32_t smem_base = c.smem_base, tmem_base = c.tmem_base;
    volatile int* const abort_flag = c.abort_flag;
    const int b = c.b, u_first = c.u_first, u_last = c.u_last;
    auto BAR = [&](int i) { return c.bar_base + 8u * (uint32_t)i; };
    const int F = p.F, n_ct = p.n_ct, T_c = p.T_c;
    int* const status = p.status;
    const uint32_t tS = tmem_base + TM_S(0, 0) + (uint32_t)x * (NBUF * SUB), tO = tmem_base + TM_O0 + (uint32_t)(x * XSV_D);
    const uint64_t qd = smem_desc(smem_base + OFF_Q + (uint32_t)x * TILE_BYTES);
    auto nsub_of = [&](int kv) {   // sub-tiles of kv tile `kv`: 1 when at most 64 of its keys exist
        const int cnt = kv < n_ct ? min(BN, T_c - kv * BN) : min(BN, F - (kv - n_ct) * BN);
        return cnt > SUB ? 2 : 1;
    };
    // S = Q K^T of sub-tile (kv tile number `it` of the CTA, half `half`) into buffer `buf`
    auto issue_qk = [&](uint32_t it, int half, uint32_t buf) {
        const uint32_t st = it % NSTAGE;
        if (half == 0) mbar_wait(BAR(B_KFULL + (int)st), (it / NSTAGE) & 1u, abort_flag, status, XSV_DEV_SITE_K);
        tc_fence_after();
        const uint64_t kd = smem_desc(smem_base + OFF_KV + st * 2 * TILE_BYTES + (uint32_t)half * (SUB * 128u));
        if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)            // 16 channels = 32 bytes inside the swizzled row
                mma_ss(tS + buf * SUB, qd + 2u * k, kd + 2u * k, IDESC_QK | fmt, k > 0);
            tc_commit(BAR(B_SFULL + x * NBUF + (int)buf));
        }
        __syncwarp();
    };
    uint32_t it0 = 0;            // kv tiles of the CTA before this unit
    uint32_t cT = 0, uT = 0;     // sub-tiles and units of this query tile before this unit
    for (int u = u_first; u <= u_last; ++u) {
        const Span sp = cta_span(p, b, u);
        if (sp.kv0 >= sp.kv1) continue;
        const int mp = u % p.npair;
        const int ntile = (mp * 2 * BM + BM < F) ? 2 : 1;
        const int n = sp.kv1 - sp.kv0;
        if (x >= ntile) {
            // This unit has no second query tile.  This warp passes the stages' barrier phases one by one and releases
            // its share of each stage: not filled again before it has, a stage never gets more than one phase ahead of
            // it, nor it of a barrier (a parity wait means nothing beyond that).
            for (int i = 0; i < n; ++i) {
                const uint32_t it = it0 + (uint32_t)i, st = it % NSTAGE;
                mbar_wait(BAR(B_KFULL + (int)st), (it / NSTAGE) & 1u, abort_flag, status, XSV_DEV_SITE_K);
                mbar_wait(BAR(B_VFULL + (int)st), (it / NSTAGE) & 1u, abort_flag, status, XSV_DEV_SITE_K);
                __syncwarp();                              // every lane has passed
                if ((threadIdx.x & 31) == 0) mbar_arrive(BAR(B_EMPTY + (int)st));
            }
            it0 += (uint32_t)n;
            continue;
        }
        mbar_wait(BAR(B_QFULL + x), uT & 1u, abort_flag, status, XSV_DEV_SITE_Q);
        tc_fence_after();
        // ---- the first NBUF QK^T of the unit
        int qi = 0, qs = 0, qj = 0;                      // next QK: kv tile of the span, half, sub-tile of the unit
        for (; qj < NBUF && qi < n; ++qj) {
            issue_qk(it0 + (uint32_t)qi, qs, (cT + (uint32_t)qj) % NBUF);
            if (qs + 1 >= nsub_of(sp.kv0 + qi)) { ++qi; qs = 0; } else ++qs;
        }
        // ---- PV(j), then QK(j + NBUF)
        int pj = 0;
        for (int i = 0; i < n; ++i) {
            const uint32_t it = it0 + (uint32_t)i, st = it % NSTAGE;
            const int ns = nsub_of(sp.kv0 + i);
            mbar_wait(BAR(B_VFULL + (int)st), (it / NSTAGE) & 1u, abort_flag, status, XSV_DEV_SITE_K);
            for (int half = 0; half < ns; ++half, ++pj) {
                const uint32_t cp = cT + (uint32_t)pj, buf = cp % NBUF;
                mbar_wait(BAR(B_PREADY + x * NBUF + (int)buf), (cp / NBUF) & 1u, abort_flag, status, XSV_DEV_SITE_P);
                tc_fence_after();
                const uint64_t vd = smem_desc(smem_base + OFF_KV + st * 2 * TILE_BYTES + TILE_BYTES + (uint32_t)half * (SUB * 128u));
                const uint32_t acc0 = pj > 0 ? 1u : 0u;
                const bool release = half + 1 == ns;          // this tile is through with the stage
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < SUB / 16; ++k)     // 16 tokens: 8 columns of P, 2048 bytes of V
                        mma_ts(tO, tS + buf * SUB + 8u * k, vd + 128u * k, IDESC_PV | fmt, k > 0 ? 1u : acc0);
                    tc_commit(BAR(B_PVDONE + x * NBUF + (int)buf));
                    if (release) tc_commit(BAR(B_EMPTY + (int)st));
                }
                __syncwarp();
                if (qi < n) {
                    issue_qk(it0 + (uint32_t)qi, qs, (cT + (uint32_t)qj) % NBUF);
                    ++qj;
                    if (qs + 1 >= nsub_of(sp.kv0 + qi)) { ++qi; qs = 0; } else ++qs;
                }
            }
        }
        it0 += (uint32_t)n;
        cT += (uint32_t)pj;
        ++uT;
    }
    // nothing of this warp's is in flight when the block ends, also where a wait ran out and no one else waits for it
    if (elect_one()) tc_commit(BAR(B_DRAIN + x));
    mbar_wait_bounded(BAR(B_DRAIN + x), 0u);
}

// ------------------------------------------------------------------ the kernel
template <typename T, int BITS, bool BF>
__global__ void __launch_bounds__(NTHREADS, 1) attn_tc5_kernel(const __grid_constant__ BatchParams bp) {
    int s_idx = 0;
    while (s_idx + 1 < bp.n && (int)blockIdx.x >= bp.cta_base[s_idx + 1]) ++s_idx;    // uniform: this CTA's stream
    const Params& p = bp.p[s_idx];
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t smem_base = smem_u32(smem);
    const uint32_t bar_base = smem_base + OFF_BAR;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + OFF_BAR + B_COUNT * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + OFF_BAR + B_COUNT * 8 + 4);
    auto BAR = [&](int i) { return bar_base + 8u * (uint32_t)i; };

    const int tid = threadIdx.x, warp = tid >> 5;
    const int b = (int)blockIdx.x - bp.cta_base[s_idx];
    const long long tick0 = cta_tick(p, b), tick1 = cta_tick(p, b + 1);
    if (tick0 >= tick1) {                             // uniform: nothing to do, nothing allocated
        xsv_dep_sync();                               // every block waits for the kernel before it, so that the order of the chain holds
        return;
    }
    const int u_first = unit_of_tick(p, tick0), u_last = unit_of_tick(p, tick1 - 1);

    if (tid == 0) {
        for (int i = 0; i < NSTAGE; ++i) {
            mbar_init(BAR(B_KFULL + i), bp.use_tma ? 1 : 4);     // one arrival per slab of 32 rows, or the one that announces the copy
            mbar_init(BAR(B_VFULL + i), bp.use_tma ? 1 : 4);
            mbar_init(BAR(B_EMPTY + i), 2);     // one per query tile: a commit, or an arrival where there is no second tile
        }
        for (int x = 0; x < 2; ++x) {
            for (int i = 0; i < NBUF; ++i) {
                mbar_init(BAR(B_SFULL + x * NBUF + i), 1);
                mbar_init(BAR(B_PREADY + x * NBUF + i), 4);     // one arrival per softmax warp
                mbar_init(BAR(B_PVDONE + x * NBUF + i), 1);
            }
            mbar_init(BAR(B_QFULL + x), 4);
            mbar_init(BAR(B_DRAIN + x), 1);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8 + NPROD + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const Cta cta{smem, smem_base, bar_base, tmem_base, abort_flag, b, u_first, u_last};

    xsv_dep_sync();      // everything above is set-up that touches no global memory
    if (warp < 8) softmax_loop<T, BITS, BF>(p, cta);
    else if (warp < 8 + NPROD) {
        if (bp.use_tma) producer_tma_loop(p, cta, bp.tm[s_idx]);
        else producer_loop<T, BITS>(p, cta);
    }
    else mma_loop(p, cta, warp - (8 + NPROD), BF ? IDESC_BF16 : 0u);
    tc_fence_before();
    __syncthreads();
    // Only now may the next kernel be scheduled: released at the start, its blocks would sit through this whole kernel
    // on whatever multiprocessor the grid leaves free (the one kept for the selection kernel of another stream).
    xsv_dep_release();
    if (warp == 8 + NPROD + 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// Merge the parts of the units that were shared by several CTAs, in CTA order.
// Grid: (16, units); block: 256 threads = 16 rows x 16 groups of 4 channels, so
// that a row's 256 bytes are read by 16 consecutive threads.
constexpr int MAX_PARTS = 256;         // a unit can be shared by as many CTAs as there are; the launcher keeps G <= MAX_PARTS
template <typename T>
__global__ void __launch_bounds__(256) attn_combine_kernel(const __grid_constant__ BatchParams bp) {
    xsv_dep_release();
    int s_idx = 0;
    while (s_idx + 1 < bp.n && (int)blockIdx.y >= bp.unit_base[s_idx + 1]) ++s_idx;
    const Params& p = bp.p[s_idx];
    __shared__ int s_slot[MAX_PARTS];
    __shared__ int s_cand[MAX_PARTS];      // per candidate CTA: -1 nothing of this unit, -2 the whole unit, else its slot
    __shared__ int s_n, s_b0, s_nb;
    const int u = (int)blockIdx.y - bp.unit_base[s_idx];
    if (threadIdx.x == 0) {
        long long base;
        int cost;
        unit_base_cost(p, u, base, cost);
        // CTAs that may hold steps of this unit
        int b0 = (int)(base * p.G / p.total), b1 = (int)((base + COST_UNIT + (long long)cost * (p.nkv - 1)) * p.G / p.total);
        b0 = max(0, b0 - 1);
        b1 = min(p.G - 1, b1 + 1);
        s_b0 = b0;
        s_nb = min(b1 - b0 + 1, MAX_PARTS);
    }
    __syncthreads();
    if (threadIdx.x < s_nb) {              // one candidate per thread: the span arithmetic is long-latency integer work
        const int b = s_b0 + threadIdx.x;
        const Span sp = cta_span(p, b, u);
        int v = -1;
        if (sp.kv0 < sp.kv1) v = (sp.kv0 == 0 && sp.kv1 == p.nkv) ? -2 : b * 2 + (sp.kv0 > 0 ? 0 : 1);
        s_cand[threadIdx.x] = v;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int n = 0;
        for (int i = 0; i < s_nb; ++i) {
            const int v = s_cand[i];
            if (v == -1) continue;
            if (v == -2) { n = 0; break; }   // whole unit in one CTA: already written
            s_slot[n++] = v;
        }
        s_n = n;
    }
    __syncthreads();
    const int n = s_n;
    xsv_dep_sync();      // the part list is arithmetic on the parameters; the parts themselves come from the attention kernel
    if (n == 0) return;  // (after the wait: every block of every kernel of the chain waits for its predecessor)
    const int h = u / p.npair, mp = u - h * p.npair;
    const int row = blockIdx.x * 16 + (threadIdx.x >> 4), c4 = threadIdx.x & 15;
    const int grow = mp * 2 * BM + row;
    if (grow >= p.F) return;
    float M = -INFINITY;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float L = 0.f;
    if (n <= 4) {
        // the usual case: every load of every part is issued before the first use (one round trip to memory)
        float2 ml[4];
        float4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ml[i] = make_float2(-INFINITY, 0.f);
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < n) {
                const float* part = p.part + (size_t)s_slot[i] * PART_STRIDE;
                ml[i] = reinterpret_cast<const float2*>(part + 256 * 64)[row];
                v[i] = reinterpret_cast<const float4*>(part + (size_t)row * 64)[c4];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) M = fmaxf(M, ml[i].x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < n) {
                const float w = exp2f(ml[i].x - M);
                L += ml[i].y * w;
                acc.x += v[i].x * w; acc.y += v[i].y * w; acc.z += v[i].z * w; acc.w += v[i].w * w;
            }
        }
    } else {
        for (int i = 0; i < n; ++i)
            M = fmaxf(M, reinterpret_cast<const float2*>(p.part + (size_t)s_slot[i] * PART_STRIDE + 256 * 64)[row].x);
        for (int i = 0; i < n; ++i) {
            const float* part = p.part + (size_t)s_slot[i] * PART_STRIDE;
            const float2 ml = reinterpret_cast<const float2*>(part + 256 * 64)[row];
            const float w = exp2f(ml.x - M);
            L += ml.y * w;
            const float4 v = reinterpret_cast<const float4*>(part + (size_t)row * 64)[c4];
            acc.x += v.x * w; acc.y += v.y * w; acc.z += v.z * w; acc.w += v.w * w;
        }
    }
    const float inv = 1.f / L;
    uint2* dst = reinterpret_cast<uint2*>(reinterpret_cast<T*>(p.out) + ((size_t)h * p.F + grow) * XSV_D) + c4;
    *dst = make_uint2(xsv_pack2<T>(acc.x * inv, acc.y * inv), xsv_pack2<T>(acc.z * inv, acc.w * inv));
}

// A wait that nothing ends: one barrier, no arrival.  Exercises the bounded wait of the attention kernel: it must
// return after WAIT_LIMIT_NS with XSV_DEV_TIMEOUT in *status instead of hanging.
__global__ void wait_selftest_kernel(int* status) {
    __shared__ uint64_t bar;
    __shared__ int abort_flag;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bar), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    mbar_wait(smem_u32(&bar), 0u, &abort_flag, status, XSV_DEV_SITE_SELFTEST);
}

template <typename T, int BITS, bool BF = false>
cudaError_t launch(const BatchParams& bp, bool merge_only, cudaStream_t st) {
    if (merge_only) {
        xsv_launch_dep(attn_combine_kernel<T>, dim3(16, bp.unit_base[bp.n]), dim3(256), 0, st, bp);
        xsv_count_launch(1);
        return cudaGetLastError();
    }
    static XsvPerDeviceInt attr_set;      // the opt-in to large dynamic shared memory holds per device
    const int dev = xsv_current_device();
    if (!attr_set.get(dev)) {
        cudaError_t e = cudaFuncSetAttribute(attn_tc5_kernel<T, BITS, BF>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<BITS>());
        if (e != cudaSuccess) return e;
        attr_set.set(dev, 1);
    }
    xsv_launch_dep(attn_tc5_kernel<T, BITS, BF>, dim3(bp.cta_base[bp.n]), dim3(NTHREADS), smem_bytes<BITS>(), st, bp);
    xsv_count_launch(1);
    return cudaGetLastError();
}

}  // namespace

cudaError_t xsv_launch_wait_selftest(int* status, cudaStream_t st) {
    wait_selftest_kernel<<<1, 64, 0, st>>>(status);
    xsv_count_launch();
    return cudaGetLastError();
}

size_t xsv_attn_tc5_workspace_bytes() { return (size_t)xsv_sm_count() * 2 * PART_STRIDE * sizeof(float); }

namespace {
// The work of one stream (everything of Params but the CTA count and the workspace slice).
void fill_params(Params& p, const LayerView& lv, int T_c, const void* Q, const void* K, const void* V, void* out, int H,
                 int F, int* status) {
    p.lv = lv; p.Q = Q; p.K = K; p.V = V; p.out = out; p.status = status;
    p.T_c = T_c; p.F = F; p.H = H;
    p.n_ct = (T_c + BN - 1) / BN;
    p.nkv = p.n_ct + (F + BN - 1) / BN;
    p.npair = (F + 2 * BM - 1) / (2 * BM);
    p.n_full = ((p.npair - 1) * 2 * BM + BM < F) ? p.npair : p.npair - 1;
    p.ticks_head = p.n_full * unit_len(p, true) + (p.npair - p.n_full) * unit_len(p, false);
    p.total = p.ticks_head * H;
}

// ---- tensor maps for the copy-engine feed (bits == 16: the cache holds the 16-bit inputs themselves)
typedef CUresult (*XsvEncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
XsvEncodeTiled encode_tiled_fn() {          // the driver's encoder, looked up once; null where there is no driver
    static XsvEncodeTiled fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (XsvEncodeTiled)f;
    }();
    return fn;
}
// [heads][rows][64] fp16 with `head_stride_rows` rows between heads, read in boxes of 128 rows; rows at or beyond
// `rows` read as zeros.  False if the tensor cannot be described (no encoder, an unaligned pointer).
bool encode_rows_map(CUtensorMap* m, const void* base, long long rows, long long head_stride_rows, int H, int dtype) {
    XsvEncodeTiled enc = encode_tiled_fn();
    if (!enc || !base || (reinterpret_cast<uintptr_t>(base) & 15u) != 0) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)XSV_D, (cuuint64_t)(rows > 0 ? rows : 1), (cuuint64_t)H};
    const cuuint64_t strides[2] = {(cuuint64_t)XSV_D * 2, (cuuint64_t)head_stride_rows * XSV_D * 2};
    const cuuint32_t box[3] = {(cuuint32_t)XSV_D, (cuuint32_t)BN, 1u};
    const cuuint32_t estr[3] = {1u, 1u, 1u};
    return enc(m, dtype == 0 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The four maps of one stream; false leaves the launch on the producers' own loads.
bool encode_stream_maps(StreamMaps& sm, const Params& p, int dtype) {
    if (p.lv.bits != 16 || p.H < 1 || p.F < 1) return false;
    return encode_rows_map(&sm.m[0], p.lv.kcodes, p.T_c, p.lv.cap, p.H, dtype) && encode_rows_map(&sm.m[1], p.lv.vcodes, p.T_c, p.lv.cap, p.H, dtype) &&
           encode_rows_map(&sm.m[2], p.K, p.F, p.F, p.H, dtype) && encode_rows_map(&sm.m[3], p.V, p.F, p.F, p.H, dtype);
}
// Whether the launch described by bp (streams and CTAs already dealt) can be fed by the copy engine, and its maps.
void prepare_tma(BatchParams& bp, int dtype) {
    static const bool off = getenv("XSV_NO_TMA") != nullptr;      // for comparisons
    bp.use_tma = 0;
    if (off || (dtype != 0 && dtype != 1) || bp.n < 1 || bp.p[0].lv.bits != 16) return;
    for (int i = 0; i < bp.n; ++i)
        if (!encode_stream_maps(bp.tm[i], bp.p[i], dtype)) return;
    bp.use_tma = 1;
}

// CTAs of the launch dealt to the streams in proportion to their work (at least one each, never more than a
// stream has steps); the CTAs of one stream then split that stream's steps among themselves as in a launch of its own.
void deal_ctas(BatchParams& bp, float* workspace, int sms) {
    long long total = 0;
    for (int i = 0; i < bp.n; ++i) total += bp.p[i].total;
    int used = 0;
    for (int i = 0; i < bp.n; ++i) {
        Params& p = bp.p[i];
        const long long steps = (long long)p.H * p.npair * p.nkv;
        long long g = total > 0 ? (p.total * sms + total / 2) / total : 1;
        const int left = sms - used - (bp.n - 1 - i);              // keep one for every stream still to come
        if (g > left) g = left;
        if (g > steps) g = steps;
        if (g > MAX_PARTS) g = MAX_PARTS;
        if (g < 1) g = 1;
        p.G = (int)g;
        p.part = workspace ? workspace + (size_t)used * 2 * PART_STRIDE : nullptr;   // no workspace: a planning call
        bp.cta_base[i] = used;
        used += p.G;
    }
    bp.cta_base[bp.n] = used;
    bp.unit_base[0] = 0;
    for (int i = 0; i < bp.n; ++i) bp.unit_base[i + 1] = bp.unit_base[i] + bp.p[i].H * bp.p[i].npair;
}

cudaError_t launch_tc5(const BatchParams& bp, int dtype, int bits, bool merge_only, cudaStream_t st) {
#define XSV_TC5(TT, B) return launch<TT, B>(bp, merge_only, st)
    if (dtype == 0) {
        switch (bits) {
            case 2: XSV_TC5(__half, 2);
            case 4: XSV_TC5(__half, 4);
            case 8: XSV_TC5(__half, 8);
            case 16: XSV_TC5(__half, 16);
        }
    } else {
        switch (bits) {
            case 2: XSV_TC5(__nv_bfloat16, 2);
            case 4: XSV_TC5(__nv_bfloat16, 4);
            case 8: XSV_TC5(__nv_bfloat16, 8);
            case 16:
                if (bp.use_tma && !merge_only) return launch<__nv_bfloat16, 16, true>(bp, merge_only, st);   // bf16 operands, copy-engine feed
                XSV_TC5(__nv_bfloat16, 16);
        }
    }
#undef XSV_TC5
    return cudaErrorInvalidValue;
}

cudaError_t launch_one(const LayerView& lv, int T_c, const void* Q, const void* K, const void* V, void* out, int dtype,
                       int H, int F, float* workspace, int* status, int spare_sms, bool merge_only, cudaStream_t st) {
    if (!workspace) return cudaErrorNotSupported;
    BatchParams bp{};
    bp.n = 1;
    fill_params(bp.p[0], lv, T_c, Q, K, V, out, H, F, status);
    const int sms = xsv_sm_count() - spare_sms > 0 ? xsv_sm_count() - spare_sms : 1;   // multiprocessors left to another kernel
    deal_ctas(bp, workspace, sms);
    if (!merge_only) prepare_tma(bp, dtype);
    return launch_tc5(bp, dtype, lv.bits, merge_only, st);
}
}  // namespace

cudaError_t xsv_launch_attn_tc5(const LayerView& lv, int T_c, const void* Q, const void* K, const void* V, void* out,
                                int dtype, int H, int F, float* workspace, int* status, int spare_sms, cudaStream_t st) {
    return launch_one(lv, T_c, Q, K, V, out, dtype, H, F, workspace, status, spare_sms, false, st);
}

cudaError_t xsv_launch_attn_tc5_merge(const LayerView& lv, int T_c, const void* Q, const void* K, const void* V,
                                      void* out, int dtype, int H, int F, float* workspace, int* status,
                                      int spare_sms, cudaStream_t st) {
    return launch_one(lv, T_c, Q, K, V, out, dtype, H, F, workspace, status, spare_sms, true, st);
}

namespace {
// CTAs do not span streams, so a launch takes as long as its slowest stream: max over the streams of ticks per CTA.
// With many streams the whole numbers of CTAs fit the work badly (eight equal streams get 18 or 19 of 148 CTAs
// each); the streams are therefore launched in consecutive groups of g, with the g among n, 4, 2, 1 whose estimated
// time -- the groups' slowest streams, plus a fixed cost per launch -- is the smallest.  Host arithmetic only.
constexpr long long LAUNCH_TICKS = 100;             // ramp and tail of a launch, in the ticks of the cost model
long long build_group(const Params* ps, int first, int count, float* workspace, int sms, BatchParams& bp) {
    bp = BatchParams{};
    bp.n = count;
    for (int i = 0; i < count; ++i) bp.p[i] = ps[first + i];
    deal_ctas(bp, workspace, sms);
    long long worst = 0;
    for (int i = 0; i < count; ++i) worst = std::max(worst, (bp.p[i].total + bp.p[i].G - 1) / bp.p[i].G);
    return worst + LAUNCH_TICKS;
}
int choose_group_size(const Params* ps, int n, int sms) {
    int best_g = n;
    long long best = -1;
    const int cand[4] = {n, 4, 2, 1};
    BatchParams bp;
    for (int c = 0; c < 4; ++c) {
        const int g = cand[c];
        if (g > n || (c > 0 && g >= cand[0])) continue;
        long long t = 0;
        for (int first = 0; first < n; first += g) t += build_group(ps, first, std::min(g, n - first), nullptr, sms, bp);
        if (best < 0 || t < best) { best = t; best_g = g; }
    }
    return best_g;
}
}  // namespace

int xsv_attn_batch_group_size(int n, const int* T_cs, const int* Fs, int H, int sms) {
    if (n < 1 || n > XSV_MAX_BATCH || sms < 1) return -1;
    Params ps[XSV_MAX_BATCH];
    const LayerView none{};
    for (int i = 0; i < n; ++i) fill_params(ps[i], none, T_cs[i], nullptr, nullptr, nullptr, nullptr, H, Fs[i], nullptr);
    return choose_group_size(ps, n, sms);
}

cudaError_t xsv_launch_attn_tc5_batch(int n, const LayerView* lvs, const int* T_cs, const void* const* Qs,
                                      const void* const* Ks, const void* const* Vs, void* const* outs, int dtype, int H,
                                      const int* Fs, float* workspace, int* const* statuses, cudaStream_t st) {
    if (!workspace || n < 1 || n > XSV_MAX_BATCH) return cudaErrorInvalidValue;
    Params ps[XSV_MAX_BATCH];
    for (int i = 0; i < n; ++i) {
        if (lvs[i].bits != lvs[0].bits) return cudaErrorInvalidValue;
        fill_params(ps[i], lvs[i], T_cs[i], Qs[i], Ks[i], Vs[i], outs[i], H, Fs[i], statuses[i]);
    }
    const int sms = xsv_sm_count();
    const int g = choose_group_size(ps, n, sms);
    BatchParams bp;
    for (int first = 0; first < n; first += g) {
        build_group(ps, first, std::min(g, n - first), workspace, sms, bp);
        prepare_tma(bp, dtype);
        cudaError_t e = launch_tc5(bp, dtype, lvs[0].bits, false, st);
        if (e != cudaSuccess) return e;
        e = launch_tc5(bp, dtype, lvs[0].bits, true, st);     // the merge reads the workspace the next group reuses
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}
