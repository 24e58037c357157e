// The record in which a page holds 64 tokens of one key/value head at 8 bits, and the device helpers of the kernels that
// read and write it.  For head_dim d a record is 130 d bytes:
//   [0, 64 d)                key codes, 16-byte pieces [8 a][d/64 c][8 g][4 j]: token 8 a + g, channels 64 c + 16 j to + 15
//   [64 d, 64 d + 12)        float32: key scale, value scale, factor of the mean key
//   [64 d + 32, 128 d + 32)  value codes, pieces of d/8 bytes [4 t][2 b][2 h][8 g][4 j]: token 16 t + 8 b + 2 j + h, channels
//                            (d/8) g to (d/8) g + d/8 - 1
//   [128 d + 32, 129 d + 32) mean key of a full page, int8 [d]
// Codes are e4m3, a value is code * scale with one scale for the block's keys and one for its values: 2^e with the smallest e
// in [-80, 8] for which 448 * 2^e reaches the largest magnitude.  A power of two costs e4m3 nothing (its steps are relative), x / 2^e
// is exact, so that the code's rounding is the only one, and so is a change of the scale until a code becomes subnormal.
// With lane = 4 g + j, 32 consecutive pieces are one 16- or 8-byte load of a warp, and what a lane then holds is its part of the
// A operand of mma.m16n8k16 (row, k) = keys: (token, channel), values: (channel, token):
//   keys:   rows g and g + 8 of tile t are tokens of a = 2 t and 2 t + 1; the k columns 2 j, 2 j + 1, 2 j + 8, 2 j + 9 of step
//           4 c + w are channels 64 c + 16 j + 4 w to + 3: a word, in order;
//   values: k columns 2 j + h and 2 j + 8 + h of step t are b = 0 and 1; rows g and g + 8 of tile i are channels (d/8) g + 2 i
//           and the one after it: bytes of two pieces, interleaved.
#pragma once
#include "page_layout.cuh"

template <int D> struct Page8Rec {
    static constexpr int K_CODES = 0, PARAMS = 64 * D, V_CODES = 64 * D + 32, MEAN = 128 * D + 32, BYTES = 130 * D;
    static constexpr int K_BYTES = 64 * D + 32, V_BYTES = 64 * D;        // keys with the parameters; values
};
constexpr int P8_EXP_MIN = -80, P8_EXP_MAX = 8;

// Checks of a pool's description, on the host; fills the kernels' view of it (no tail).
xsv_status xsv_page8_view(const xsv_page8_pool* pool, PoolView* v);       // page8_cache.cu

template <int D> __device__ __forceinline__ uint8_t* page8_rec(const PoolView& pv, int page, int head) {
    return pv.rec + ((size_t)page * pv.heads + head) * Page8Rec<D>::BYTES;
}
__device__ __forceinline__ float p8_pow2(int e) { return __int_as_float((e + 127) << 23); }              // e in [-126, 127]
// Exponent for a largest magnitude (at most 65536): 448 is 1.75 * 2^8.
__device__ __forceinline__ int p8_exponent(float amax) {
    const int bits = __float_as_int(amax);
    const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
    return min(max(e, P8_EXP_MIN), P8_EXP_MAX);
}
// Exponent of a scale that stands in a record.
__device__ __forceinline__ int p8_exponent_of(float scale) { return min(max((__float_as_int(scale) >> 23 & 0xFF) - 127, P8_EXP_MIN), P8_EXP_MAX); }
// two floats -> two e4m3 codes, nearest-even, the first in the low byte
__device__ __forceinline__ uint32_t p8_codes2(float lo, float hi) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// the two codes in the low or high half of a word -> fp16 pair (every e4m3 value is one)
__device__ __forceinline__ void p8_halves(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
