// The record in which a page holds 64 tokens of one key/value head at 4 bits, and the device helpers of the kernels
// that read and write it.  For head_dim d a record is 72 d bytes:
//   [0, 32 d)     key codes    [d/16 k][8 g][4 j][4 m] 32-bit words
//   [32 d, 64 d)  value codes  [4 k][d/64 c][8 g][4 j][4 m] 32-bit words
//   [64 d, 72 d)  fp16: key scale [d], key offset [d], value scale [d/64][8 g][8 i], value offset [d/64][8 g][8 i]
//                 (token 8 i + g)
// A word is one lane's A operand of mma.m16n8k16 (row, k) = keys: (token, channel), values: (channel, token), with
// lane = 4 g + j: nibbles 0..7 are, from the low end,
//   (g, lo0) (g + 8, lo0) (g, hi0) (g + 8, hi0) (g, lo1) (g + 8, lo1) (g, hi1) (g + 8, hi1)
// where lo = k columns 2 j + {0, 1} and hi = 2 j + 8 + {0, 1}.  Masking with 0x000F000F therefore yields the fp16 pair
// of an operand register as subnormals, code * 2^-24, and with 0x00F000F0 that of the row eight below as
// code * 2^-20: no subtraction and no conversion, one logic operation per two codes; the powers of two are taken
// out of the float32 accumulator, where each row has its own.
//   keys:   row r of word m is token 16 m + r; column 2 j + {0, 1} of step k is channel 32 (k/2) + 8 j + 4 (k%2) + {0, 1},
//           column 2 j + 8 + {0, 1} the two after it: a lane's channels are 8 consecutive ones per two steps, so that
//           a row of 16-bit queries or keys is read 16 bytes at a time;
//   values: column r of step k is token 16 k + r; row g of word m is channel 64 c + 8 g + 2 m, row g + 8 the one after
//           it: a lane's output channels are 8 consecutive ones.
// Scales and offsets are fp16, rounded outwards (offset down, scale up), so that no value leaves the code range and a
// value is off by at most half a scale.  Where the last code would stand for more than 65504 the scale is rounded down
// instead, so that every value is a finite fp16: the maximum is then off by at most 15 steps of s, 2^-10 s each.
#pragma once
#include "../../include/xsv.h"
#include "xsv_common.cuh"

#define XSV_PAGE XSV_PAGE_TOKENS

template <int D> struct PageRec {
    static constexpr int K_CODES = 0, V_CODES = 32 * D, K_SCALE = 64 * D, K_ZERO = 66 * D, V_SCALE = 68 * D,
                         V_ZERO = 70 * D, BYTES = 72 * D;
};

// The pool as the kernels see it (host struct xsv_page_pool).
struct PoolView {
    uint8_t* rec;
    void* k_tail;        // [max_seqs][2][heads][64][d], 16-bit
    long long n_pages;
    int max_seqs, heads;
};

// Checks of a pool's description, on the host; fills the kernels' view of it.
xsv_status xsv_pool_view(const xsv_page_pool* pool, PoolView* v);   // page_cache.cu
// Turns a CUDA error into XSV_ERR_CUDA and keeps it for xsv_last_cuda_error.
xsv_status xsv_cuda_status(cudaError_t e);                          // xsv_api.cu

template <typename T, int D> __device__ __forceinline__ T* tail_rows(const PoolView& pv, int seq, int page, int head) {
    return static_cast<T*>(pv.k_tail) + ((((size_t)seq * 2 + (page & 1)) * pv.heads + head) * XSV_PAGE) * D;
}
template <int D> __device__ __forceinline__ uint8_t* page_rec(const PoolView& pv, int page, int head) {
    return pv.rec + ((size_t)page * pv.heads + head) * PageRec<D>::BYTES;
}

// two 16-bit values of a word as floats
template <typename T> __device__ __forceinline__ float2 xsv_unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 xsv_unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
template <> __device__ __forceinline__ float2 xsv_unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

// Scale and offset of a group from its minimum and maximum (already inside +-65504).  The offset is the minimum rounded
// down to fp16; the scale is the smallest fp16 whose 15-fold (exact in float32) reaches the maximum minus the offset: the
// nearest fp16 to a fifteenth of that difference (rounded up), or the next one; and the one below where that 15-fold is
// beyond 65504 minus the offset (which the one below never is: it does not reach the maximum).
__device__ __forceinline__ void page_params(float mn, float mx, __half& s, __half& z) {
    z = __float2half_rd(mn);
    const float d = __fsub_ru(mx, __half2float(z));
    s = __float2half_rn(d * 0.066666670f);
    unsigned short bits = __half_as_ushort(s);
    if (__half2float(s) * 15.f < d) ++bits;
    if (__half2float(__ushort_as_half(bits)) * 15.f > __fsub_rd(65504.f, __half2float(z))) --bits;
    s = __ushort_as_half(bits ? bits : (unsigned short)0x3C00);       // 1 for a group of one value
}
__device__ __forceinline__ float page_inverse(float s) {            // within 2^-23
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return r;
}
// Codes of 8 values with the same parameters: nearest-even of the quotients (x - z) / s.  A quotient is inside
// [0, 15 + 2^-6] (outward rounding: 15 + 2^-19); (x - z) * inv is within 2^-18 of it.  Where that is nowhere within 2e-5 of a half-integer its
// rounding (1.5 * 2^23 added: the integer is in the low bits) is the quotient's; else the remainders of all eight decide, which
// are exact next to a half-integer.  The mask keeps an infinite or NaN value from its neighbours in a code word.
__device__ __forceinline__ void page_codes(const float (&x)[8], float s, float inv, float z, uint32_t (&c)[8]) {
    float d[8], near = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        d[i] = __fsub_rn(x[i], z);
        const float y = __fmul_rn(d[i], inv), t = __fadd_rn(y, 12582912.f);
        near = fmaxf(near, fabsf(__fsub_rn(y, __fadd_rn(t, -12582912.f))));
        c[i] = __float_as_uint(t);
    }
    if (near > 0.49998f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float k = __fadd_rn(__uint_as_float(c[i]), -12582912.f), r2 = 2.f * fmaf(-k, s, d[i]);
            if (fabsf(r2) > s || (fabsf(r2) == s && (c[i] & 1u))) c[i] += r2 > 0.f ? 1u : 0xFFFFFFFFu;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] &= 15u;
}
// minimum and maximum of pairs of 16-bit values
template <typename T> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b);
template <typename T> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t min2<__half>(uint32_t a, uint32_t b) { uint32_t d; asm("min.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
template <> __device__ __forceinline__ uint32_t max2<__half>(uint32_t a, uint32_t b) { uint32_t d; asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
template <> __device__ __forceinline__ uint32_t min2<__nv_bfloat16>(uint32_t a, uint32_t b) { uint32_t d; asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
template <> __device__ __forceinline__ uint32_t max2<__nv_bfloat16>(uint32_t a, uint32_t b) { uint32_t d; asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
__device__ __forceinline__ float clamp_half(float x) { return fminf(fmaxf(x, -65504.f), 65504.f); }

// Where new token t of an append lands.  False for a token without a place, or with one that contradicts the lengths.
struct PagePlace { int seq, begin, end, page, off, pos; };
__device__ __forceinline__ bool page_place(const int* slot_map, const int* token_seq, const int* cu, const int* total, int n_tokens, int n_seqs,
                                           long long n_pages, int t, PagePlace& q) {
    const int slot = slot_map[t];
    q.seq = token_seq[t];
    if (slot < 0 || q.seq < 0 || q.seq >= n_seqs) return false;
    q.begin = cu[q.seq];
    q.end = cu[q.seq + 1];
    q.page = slot / XSV_PAGE;
    q.off = slot % XSV_PAGE;
    if (q.begin < 0 || q.begin > t || q.end <= t || q.end > n_tokens || q.page >= n_pages) return false;
    q.pos = total[q.seq] - (q.end - t);
    return q.pos >= q.off && q.pos - (t - q.begin) >= 0 && q.pos % XSV_PAGE == q.off;
}
