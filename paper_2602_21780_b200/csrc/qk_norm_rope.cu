// Queries and keys of a projection -> normalised per head, rotated by position, laid out for the attention; values
// only laid out.  One pass: y = norm(x) * w + b over the head's channels, then (lo, hi) -> (lo cos a - hi sin a,
// hi cos a + lo sin a) with a = position * inv_freq.
//
// Bound by HBM: 2 bytes read and 2 written per element, about 10 float32 operations.  A head's row is held by d / 8
// lanes, 8 channels each as two 8-byte pieces that are partners in the rotation (for half-split and 2-D rotation the
// pieces lie half a rotated span apart), so the rotation needs no exchange between lanes; the norm's sum takes
// log2(d / 8) shuffles.  A block serves one token: its first threads compute the token's cosines and sines once, in
// shared memory, for all its heads; each lane group has two rows in flight.  With few tokens a token's heads are
// spread over several blocks (a row per lane group), which trades repeated sines for latency.
//
// Angles: position * inv_freq in turns as a float64 product, its fraction in float32: a float32 angle of a position
// near 10^6 would be off by 0.03 rad.  Norms are float32, the layer norm's variance from differences to the mean (two
// passes over registers); results are rounded once, to the output type.
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

template <typename T> __device__ __forceinline__ void load4(const T* p, float (&o)[4]) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    const float2 a = xsv_unpack2<T>(w.x), b = xsv_unpack2<T>(w.y);
    o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
}

template <typename T, int D, int ROPE>
__global__ void __launch_bounds__(128) qk_norm_rope_kernel(const __grid_constant__ NormRope p, int norm, int rows_per_group) {
    constexpr int L = D / 8, GROUPS = 128 / L;
    __shared__ float2 cs[D / 2];
    xsv_dep_release();
    xsv_dep_sync();
    const int t = blockIdx.x, lane = threadIdx.x % L, group = threadIdx.x / L;
    if (ROPE != XSV_ROPE_NONE) {
        // frequency f of the token: a span of n_rot channels for one position, two half-width spans for two
        const int n = p.n_rot / 2;
        if ((int)threadIdx.x < n) {
            const int per = ROPE == XSV_ROPE_2D ? n / 2 : n, f = threadIdx.x % per;
            const int at = ROPE == XSV_ROPE_2D ? p.pos[2 * (size_t)t + threadIdx.x / per] : p.pos[t];
            double turns = (double)at * (double)p.inv_freq[f] * 0.15915494309189533577;
            turns -= rint(turns);
            float s, c;
            sincospif(2.f * (float)turns, &s, &c);
            cs[threadIdx.x] = make_float2(c, s);
        }
        __syncthreads();
    }
    // the lane's two pieces of four channels, and the index of the first frequency of each pair it rotates
    int ca, cb, f;
    bool rot;
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
    float w[2][8], b[2][8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { w[s][i] = 1.f; b[s][i] = 0.f; }
        if (norm != XSV_NORM_NONE && p.w[s]) {
            load4<T>((const T*)p.w[s] + ca, reinterpret_cast<float(&)[4]>(w[s][0]));
            load4<T>((const T*)p.w[s] + cb, reinterpret_cast<float(&)[4]>(w[s][4]));
        }
        if (norm != XSV_NORM_NONE && p.b[s]) {
            load4<T>((const T*)p.b[s] + ca, reinterpret_cast<float(&)[4]>(b[s][0]));
            load4<T>((const T*)p.b[s] + cb, reinterpret_cast<float(&)[4]>(b[s][4]));
        }
    }
    float2 r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = rot ? cs[f + i] : make_float2(1.f, 0.f);

    const int hq = p.heads[0], hk = hq + p.heads[1], hall = hk + p.heads[2];
    const int first = (blockIdx.y * rows_per_group) * GROUPS + group;
    auto locate = [&](int h, int& part, int& head) {
        part = h < hq ? 0 : h < hk ? 1 : 2;
        head = h - (part == 0 ? 0 : part == 1 ? hq : hk);
    };
    auto fetch = [&](int h, uint2& a, uint2& c) {
        int part, head;
        locate(h, part, head);
        const T* src = (const T*)p.x[part] + (size_t)t * p.stride[part] + (size_t)head * D;
        a = *reinterpret_cast<const uint2*>(src + ca);
        c = *reinterpret_cast<const uint2*>(src + cb);
    };
    uint2 na = make_uint2(0, 0), nb = na;
    if (first < hall) fetch(first, na, nb);
    for (int k = 0; k < rows_per_group; ++k) {
        const int h = first + k * GROUPS;
        if (h - group >= hall) break;                       // the same for the whole block
        const bool live = h < hall;
        const uint2 a = na, c = nb;
        if (k + 1 < rows_per_group && h + GROUPS < hall) fetch(h + GROUPS, na, nb);
        int part = 0, head = 0;
        locate(live ? h : 0, part, head);
        uint2 oa = a, oc = c;
        float v[8];
        {
            const float2 q0 = xsv_unpack2<T>(a.x), q1 = xsv_unpack2<T>(a.y), q2 = xsv_unpack2<T>(c.x), q3 = xsv_unpack2<T>(c.y);
            v[0] = q0.x; v[1] = q0.y; v[2] = q1.x; v[3] = q1.y; v[4] = q2.x; v[5] = q2.y; v[6] = q3.x; v[7] = q3.y;
        }
        if (norm != XSV_NORM_NONE) {
            // every lane of the warp takes part in the shuffles, whatever its row
            float mean = 0.f;
            if (norm == XSV_NORM_LAYER) {
#pragma unroll
                for (int i = 0; i < 8; ++i) mean += v[i];
#pragma unroll
                for (int o = L / 2; o > 0; o >>= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);
                mean *= 1.f / D;
            }
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) { v[i] -= mean; ss = fmaf(v[i], v[i], ss); }
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
            const float inv = 1.f / sqrtf(ss * (1.f / D) + p.eps);
            const int s = part == 1;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i] * inv, s ? w[1][i] : w[0][i], s ? b[1][i] : b[0][i]);
        }
        if (part < 2) {
            if (rot) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float& lo = ROPE == XSV_ROPE_PAIRS ? v[2 * i] : v[i];
                    float& hi = ROPE == XSV_ROPE_PAIRS ? v[2 * i + 1] : v[4 + i];
                    const float x0 = lo, x1 = hi;
                    lo = x0 * r[i].x - x1 * r[i].y;
                    hi = x1 * r[i].x + x0 * r[i].y;
                }
            }
            oa = make_uint2(xsv_pack2<T>(v[0], v[1]), xsv_pack2<T>(v[2], v[3]));
            oc = make_uint2(xsv_pack2<T>(v[4], v[5]), xsv_pack2<T>(v[6], v[7]));
        }
        if (live) {
            T* dst = (T*)p.y[part] + (size_t)t * p.y_tok[part] + (size_t)head * p.y_head[part];
            *reinterpret_cast<uint2*>(dst + ca) = oa;
            *reinterpret_cast<uint2*>(dst + cb) = oc;
        }
    }
}

template <typename T, int D>
cudaError_t launch(const NormRope& p, int norm, int rope, cudaStream_t st) {
    const int groups = 128 / (D / 8), hall = p.heads[0] + p.heads[1] + p.heads[2];
    const int each = (hall + groups - 1) / groups;          // rows per lane group if one block serves a token
    // Below two blocks per multiprocessor the heads are spread over blocks as well.
    const int rows = (long long)p.n_tokens >= 2LL * xsv_sm_count() ? each : 1;
    const dim3 grid(p.n_tokens, (each + rows - 1) / rows);
    auto go = [&](auto kernel) { return xsv_launch_dep(kernel, grid, dim3(128), 0, st, p, norm, rows); };
    switch (rope) {
        case XSV_ROPE_HALF: return go(qk_norm_rope_kernel<T, D, XSV_ROPE_HALF>);
        case XSV_ROPE_PAIRS: return go(qk_norm_rope_kernel<T, D, XSV_ROPE_PAIRS>);
        case XSV_ROPE_2D: return go(qk_norm_rope_kernel<T, D, XSV_ROPE_2D>);
        default: return go(qk_norm_rope_kernel<T, D, XSV_ROPE_NONE>);
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
