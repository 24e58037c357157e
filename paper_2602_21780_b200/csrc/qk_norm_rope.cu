// Queries and keys of a projection -> normalised per head, rotated by position, laid out for the attention; values
// only laid out.  One pass: y = norm(x) * w + b over the head's channels, then (lo, hi) -> (lo cos a - hi sin a,
// hi cos a + lo sin a) with a = position * inv_freq.
//
// Bound by HBM: 2 bytes read and 2 written per element, about 10 float32 operations.  A head's row is held by d / 8
// lanes, 8 channels each as two 8-byte pieces that are partners in the rotation (for half-split and 2-D rotation the
// pieces lie half a rotated span apart), so the rotation needs no exchange between lanes; the norm's sum takes
// log2(d / 8) shuffles.  A block walks through tokens: its first threads compute a token's cosines and sines once, in
// shared memory, for all its heads; q, k and v of a token follow one another, with up to two rows of a lane group in
// flight (one where a part has no more heads than the block has lane groups: 8 of 128 channels, 16 of 64).  With few
// tokens a token's heads are spread over several blocks (a row per lane group), which trades repeated sines for latency.
//
// Angles: position * inv_freq in turns as a float64 product, its fraction in float32: a float32 angle of a position
// near 10^6 would be off by 0.03 rad.  Norms are float32, the layer norm's variance from differences to the mean (two
// passes over registers); results are rounded once, to the output type.
// Measured: 8191 tokens, 32 + 8 + 8 heads of 128, fp16: 43.6 us, 4.6 TB/s; 1374 tokens, 3 x 16 heads of 64: 6.2 us; one token: 2.5 us.
// What is left to the copy rate is loads in flight: 8 blocks of 4 warps with one or two rows each; four rows a lane group or fewer
// blocks were slower (48-52 us), and packed float32 arithmetic changed nothing.
#include <algorithm>
#include <type_traits>

#include "../../include/xsv.h"
#include "page_layout.cuh"
#include "xsv_kernels.h"

namespace {

struct NormRope {
    const void* x[3];        // q, k, v rows
    long long stride[3];     // elements from token to token
    void* y[3];
    long long y_tok[3], y_head[3];
    int heads[3];
    const void* w[2];
    const void* b[2];
    const float* inv_freq;
    const int* pos;
    float eps;
    int n_tokens, n_rot;     // n_rot: channels rotated (0: none)
};

template <typename T> __device__ __forceinline__ void unpack4(const uint2& w, float* o) {
    const float2 a = xsv_unpack2<T>(w.x), b = xsv_unpack2<T>(w.y);
    o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
}

constexpr int THREADS = 128, FLIGHT = 2;      // FLIGHT: rows of a lane group in flight

template <typename T, int D, int ROPE, int NORM, bool BIAS>
__global__ void __launch_bounds__(THREADS, 8) qk_norm_rope_kernel(const __grid_constant__ NormRope p) {
    constexpr int L = D / 8, GROUPS = THREADS / L;
    __shared__ float2 cs[2][D / 2];
    xsv_dep_release();
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    // the lane's two pieces of four channels, and the index of the first frequency of each pair it rotates
    int ca, cb, f = 0;
    bool rot = false;
    if (ROPE == XSV_ROPE_PAIRS || ROPE == XSV_ROPE_NONE) {
        ca = 8 * lane; cb = ca + 4; f = 4 * lane; rot = ROPE != XSV_ROPE_NONE && ca < p.n_rot;
    } else {
        const int span = ROPE == XSV_ROPE_2D ? D / 2 : p.n_rot, half = span / 2, lanes = span / 8;
        const int part = ROPE == XSV_ROPE_2D ? lane / lanes : 0, i = lane - part * lanes;
        rot = ROPE == XSV_ROPE_2D || lane < lanes;
        ca = rot ? part * span + 4 * i : 8 * lane;
        cb = rot ? ca + half : ca + 4;
        f = part * half + 4 * i;
    }
    xsv_dep_sync();
    uint2 wgt[2][2], bias[2][2];                            // [q, k][piece], 16-bit; BIAS: there is one (its registers cost 7 %)
    if (NORM != XSV_NORM_NONE) {
        const uint32_t one = xsv_pack2<T>(1.f, 1.f);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            wgt[s][0] = wgt[s][1] = make_uint2(one, one);
            bias[s][0] = bias[s][1] = make_uint2(0u, 0u);
            if (p.w[s]) {
                wgt[s][0] = *reinterpret_cast<const uint2*>((const T*)p.w[s] + ca);
                wgt[s][1] = *reinterpret_cast<const uint2*>((const T*)p.w[s] + cb);
            }
            if (BIAS && p.b[s]) {
                bias[s][0] = *reinterpret_cast<const uint2*>((const T*)p.b[s] + ca);
                bias[s][1] = *reinterpret_cast<const uint2*>((const T*)p.b[s] + cb);
            }
        }
    }
    const int n_freq = p.n_rot / 2, h0 = blockIdx.y * GROUPS, step = gridDim.y * GROUPS;
    // the frequency this thread serves; its position is fetched a token ahead
    const bool serves = ROPE != XSV_ROPE_NONE && (int)threadIdx.x < n_freq;
    int coord = 0, at = 0;
    double freq = 0.0;
    if (serves) {
        const int per = ROPE == XSV_ROPE_2D ? n_freq / 2 : n_freq;
        coord = threadIdx.x / per;
        freq = (double)p.inv_freq[threadIdx.x - coord * per];
        at = ROPE == XSV_ROPE_2D ? p.pos[2 * (size_t)blockIdx.x + coord] : p.pos[blockIdx.x];
    }
    int buf = 0;
    for (int t = blockIdx.x; t < p.n_tokens; t += gridDim.x, buf ^= 1) {
        float2 r[4];
        if (ROPE != XSV_ROPE_NONE) {
            if (serves) {
                double turns = (double)at * freq * 0.15915494309189533577;
                turns -= rint(turns);
                float s, c;
                sincospif(2.f * (float)turns, &s, &c);
                cs[buf][threadIdx.x] = make_float2(c, s);
                const int next = t + gridDim.x;
                if (next < p.n_tokens) at = ROPE == XSV_ROPE_2D ? p.pos[2 * (size_t)next + coord] : p.pos[next];
            }
            __syncthreads();                                // two buffers: the last token's are read before this one
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = rot ? cs[buf][f + i] : make_float2(1.f, 0.f);
        }
#pragma unroll
        for (int part = 0; part < 3; ++part) {
            const int heads = p.heads[part];
            if (h0 >= heads) continue;
            const T* src = (const T*)p.x[part] + (size_t)t * p.stride[part];
            T* dst = (T*)p.y[part] + (size_t)t * p.y_tok[part];
            float w[8], b[8];
            if (NORM != XSV_NORM_NONE && part < 2) {
                unpack4<T>(wgt[part][0], w); unpack4<T>(wgt[part][1], w + 4);
                if (BIAS) { unpack4<T>(bias[part][0], b); unpack4<T>(bias[part][1], b + 4); }
            }
            // two rows of the group at a time; every lane of the warp takes part in the shuffles, whatever its row
            for (int base = h0; base < heads; base += FLIGHT * step) {
                uint2 in[FLIGHT][2];
#pragma unroll
                for (int u = 0; u < FLIGHT; ++u) {
                    const int h = base + u * step + group;
                    in[u][0] = in[u][1] = make_uint2(0u, 0u);
                    if (h < heads) {
                        in[u][0] = *reinterpret_cast<const uint2*>(src + (size_t)h * D + ca);
                        in[u][1] = *reinterpret_cast<const uint2*>(src + (size_t)h * D + cb);
                    }
                }
#pragma unroll
                for (int u = 0; u < FLIGHT; ++u) {
                    const int h = base + u * step + group;
                    if (base + u * step >= heads) break;    // the same for the whole block
                    if (part < 2 && (NORM != XSV_NORM_NONE || ROPE != XSV_ROPE_NONE)) {
                        float v[8];
                        unpack4<T>(in[u][0], v);
                        unpack4<T>(in[u][1], v + 4);
                        if (NORM != XSV_NORM_NONE) {
                            if (NORM == XSV_NORM_LAYER) {
                                float mean = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
#pragma unroll
                                for (int o = L / 2; o > 0; o >>= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);
                                mean *= 1.f / D;
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[i] -= mean;
                            }
                            float ss = 0.f;
#pragma unroll
                            for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
#pragma unroll
                            for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
                            const float inv = rsqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = BIAS ? fmaf(v[i] * inv, w[i], b[i]) : v[i] * inv * w[i];
                        }
                        if (ROPE != XSV_ROPE_NONE) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float& lo = ROPE == XSV_ROPE_PAIRS ? v[2 * i] : v[i];
                                float& hi = ROPE == XSV_ROPE_PAIRS ? v[2 * i + 1] : v[4 + i];
                                const float x0 = lo, x1 = hi;
                                lo = x0 * r[i].x - x1 * r[i].y;
                                hi = x1 * r[i].x + x0 * r[i].y;
                            }
                        }
                        in[u][0] = make_uint2(xsv_pack2<T>(v[0], v[1]), xsv_pack2<T>(v[2], v[3]));
                        in[u][1] = make_uint2(xsv_pack2<T>(v[4], v[5]), xsv_pack2<T>(v[6], v[7]));
                    }
                    if (h < heads) {
                        T* to = dst + (size_t)h * p.y_head[part];
                        *reinterpret_cast<uint2*>(to + ca) = in[u][0];
                        *reinterpret_cast<uint2*>(to + cb) = in[u][1];
                    }
                }
            }
        }
    }
}

template <typename T, int D>
cudaError_t launch(const NormRope& p, int norm, int rope, cudaStream_t st) {
    const int groups = THREADS / (D / 8), most = std::max(p.heads[0], std::max(p.heads[1], p.heads[2])), full = 8 * xsv_sm_count();
    // With few tokens their heads are spread over several blocks as well, a row per lane group; with many a block walks
    // through its share of them (32 + 8 + 8 heads of 128: 148 tokens 3.1 against 3.6 us, 296 tokens 3.9 either way, 592
    // tokens 5.8 against 4.4).
    const dim3 grid(std::min(p.n_tokens, full), p.n_tokens >= 2 * xsv_sm_count() ? 1 : (most + groups - 1) / groups);
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, grid, dim3(THREADS), 0, st, p); };
    const bool bias = p.b[0] || p.b[1];
    auto with = [&](auto rope_c) {
        constexpr int ROPE = decltype(rope_c)::value;
        switch (norm) {
            case XSV_NORM_RMS: return bias ? go(qk_norm_rope_kernel<T, D, ROPE, XSV_NORM_RMS, true>) : go(qk_norm_rope_kernel<T, D, ROPE, XSV_NORM_RMS, false>);
            case XSV_NORM_LAYER: return bias ? go(qk_norm_rope_kernel<T, D, ROPE, XSV_NORM_LAYER, true>) : go(qk_norm_rope_kernel<T, D, ROPE, XSV_NORM_LAYER, false>);
            default: return go(qk_norm_rope_kernel<T, D, ROPE, XSV_NORM_NONE, false>);
        }
    };
    switch (rope) {
        case XSV_ROPE_HALF: return with(std::integral_constant<int, XSV_ROPE_HALF>{});
        case XSV_ROPE_PAIRS: return with(std::integral_constant<int, XSV_ROPE_PAIRS>{});
        case XSV_ROPE_2D: return with(std::integral_constant<int, XSV_ROPE_2D>{});
        default: return with(std::integral_constant<int, XSV_ROPE_NONE>{});
    }
}

}  // namespace


extern "C" xsv_status xsv_qk_norm_rope(const void* q, const void* k, const void* v, long long q_stride, long long k_stride,
                                       long long v_stride, int n_tokens, int q_heads, int kv_heads, int head_dim,
                                       xsv_dtype dtype, xsv_norm norm, const void* q_weight, const void* q_bias,
                                       const void* k_weight, const void* k_bias, float eps, xsv_rope rope, int rotary_dim,
                                       const float* inv_freq, const int* positions, xsv_layout layout, void* q_out,
                                       void* k_out, void* v_out, void* stream) {
    if (n_tokens < 0 || q_heads < 0 || kv_heads < 0 || q_heads > 1 << 16 || kv_heads > 1 << 16) return XSV_ERR_ARG;
    if (head_dim != 64 && head_dim != 128) return XSV_ERR_ARG;
    if (dtype != XSV_F16 && dtype != XSV_BF16) return XSV_ERR_ARG;
    if ((int)norm < XSV_NORM_NONE || (int)norm > XSV_NORM_LAYER || (int)rope < XSV_ROPE_NONE || (int)rope > XSV_ROPE_2D) return XSV_ERR_ARG;
    if (layout != XSV_TOKEN_MAJOR && layout != XSV_HEAD_MAJOR) return XSV_ERR_ARG;
    if (!(eps >= 0.f)) return XSV_ERR_ARG;
    if (n_tokens == 0) return XSV_OK;
    const void* in[3] = {q, k, v};
    void* out[3] = {q_out, k_out, v_out};
    const long long stride[3] = {q_stride, k_stride, v_stride};
    uintptr_t bits = 0;
    NormRope p{};
    for (int i = 0; i < 3; ++i) {
        if ((in[i] == nullptr) != (out[i] == nullptr)) return XSV_ERR_ARG;
        const int heads = !in[i] ? 0 : i == 0 ? q_heads : kv_heads;
        if (in[i] && heads == 0) return XSV_ERR_ARG;
        if (in[i] && n_tokens > 1 && stride[i] < (long long)heads * head_dim) return XSV_ERR_ARG;
        if (in[i] && (stride[i] & 7)) return XSV_ERR_SHAPE;
        bits |= (uintptr_t)in[i] | (uintptr_t)out[i];
        p.x[i] = in[i]; p.y[i] = out[i]; p.stride[i] = stride[i]; p.heads[i] = heads;
        p.y_tok[i] = layout == XSV_TOKEN_MAJOR ? (long long)heads * head_dim : head_dim;
        p.y_head[i] = layout == XSV_TOKEN_MAJOR ? head_dim : (long long)n_tokens * head_dim;
    }
    if (!q && !k && !v) return XSV_ERR_ARG;
    if (rope != XSV_ROPE_NONE) {
        if (!inv_freq || !positions || rotary_dim <= 0 || rotary_dim > head_dim || rotary_dim % 8) return XSV_ERR_ARG;
        if (rope == XSV_ROPE_2D && rotary_dim != head_dim) return XSV_ERR_ARG;
        if (((uintptr_t)inv_freq | (uintptr_t)positions) & 3) return XSV_ERR_SHAPE;
    }
    if (norm != XSV_NORM_NONE) bits |= (uintptr_t)q_weight | (uintptr_t)q_bias | (uintptr_t)k_weight | (uintptr_t)k_bias;
    if (bits & 15) return XSV_ERR_SHAPE;
    p.w[0] = q_weight; p.w[1] = k_weight; p.b[0] = q_bias; p.b[1] = k_bias;
    p.inv_freq = inv_freq; p.pos = positions; p.eps = eps; p.n_tokens = n_tokens;
    p.n_rot = rope == XSV_ROPE_NONE ? 0 : rotary_dim;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (dtype == XSV_F16) e = head_dim == 64 ? launch<__half, 64>(p, norm, rope, st) : launch<__half, 128>(p, norm, rope, st);
    else e = head_dim == 64 ? launch<__nv_bfloat16, 64>(p, norm, rope, st) : launch<__nv_bfloat16, 128>(p, norm, rope, st);
    if (e != cudaSuccess) return xsv_cuda_status(e);
    xsv_count_launch(1);
    return XSV_OK;
}
