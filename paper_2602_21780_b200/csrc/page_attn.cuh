// What the attention kernels over pages share: the arguments, and a sequence as both split it.
#pragma once
#include "page_layout.cuh"
#include "tc5_ptx.cuh"

struct PageAttn {
    PoolView pool;
    const void* Q;
    void* out;
    const int* table;
    const int* cu;
    const int* total;
    const int* slot;     // the plan's, or null: says which sequences it refused
    long long q_stride;
    float scale;         // times log2 e
    int width, n_seqs, n_tokens, q_heads, group, window;
    int group_shift;     // log2 of group where it is a power of two, else -1
    int row_limit;       // sequences of at most so many query rows a head go to the kernel for few rows, the others to
                         // the one for many
};

// total: tokens that the table row has pages for; first: position of the first new token, which may lie beyond them
struct PageSeq { int new_, total, first; };
__device__ __forceinline__ PageSeq page_seq(const PageAttn& p, int s) {
    PageSeq q;
    const int a = min(max(p.cu[s], 0), p.n_tokens), b = min(max(p.cu[s + 1], a), p.n_tokens);
    q.new_ = b - a;
    int held = max(p.total[s], 0);
    // A refused sequence still holds what it held, but its new tokens are not among it: they see nothing.
    if (p.slot && b > a && p.slot[a] < 0) held = 0;
    q.total = min(held, p.width * XSV_PAGE);
    q.first = held - q.new_;
    return q;
}
constexpr float MIN_FACTOR = 1.17549435e-38f;     // a logit factor does not underflow: times a masked place's -infinity, 0 would be NaN

// Two results -> 16 bits.  Results are means of values of at most 65504, but the rounding of the weights may carry one
// past the largest fp16.  A NaN stays.
template <typename T> __device__ __forceinline__ uint32_t page_result2(float a, float b) { return xsv_pack2<T>(a, b); }
template <> __device__ __forceinline__ uint32_t page_result2<__half>(float a, float b) {
    auto in = [](float x) {
        asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(65504.f));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(-65504.f));
        return x;
    };
    return xsv_pack2<__half>(in(a), in(b));
}
// query row of a key/value head -> new token and query head of the group
__device__ __forceinline__ void page_row(const PageAttn& p, int r, int& i, int& h) {
    i = p.group_shift >= 0 ? r >> p.group_shift : r / p.group;
    h = r - i * p.group;
}

// The kernel for many rows (page_attn_tc5.cu): work list, attention, merge.
size_t xsv_page_tc5_workspace(int n_tokens, int n_seqs, int group, int head_dim);
cudaError_t xsv_launch_page_tc5(const PageAttn& p, xsv_dtype dtype, int head_dim, void* workspace, cudaStream_t st);
cudaError_t xsv_launch_page8_tc5(const PageAttn& p, xsv_dtype dtype, int head_dim, void* workspace, cudaStream_t st);     // over 8-bit pages

// ------------------------------------------------------------------ mma.sync and register helpers
namespace {
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// c = a b
__device__ __forceinline__ void mma0(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// d = a b + c
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const float (&c)[4]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1),
                   "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t hmul2_u(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
// halves i of two 8-half vectors as a pair
__device__ __forceinline__ uint32_t pair_at(const uint4& a, const uint4& b, int i) {
    return __byte_perm(word(a, i >> 1), word(b, i >> 1), i & 1 ? 0x7632 : 0x5410);
}
__device__ __forceinline__ float pow2i(int e) {            // 2^e, clamped to what float32 holds as a normal number
    return __int_as_float((min(max(e, -126), 127) + 127) << 23);
}
constexpr size_t align256(size_t v) { return (v + 255) / 256 * 256; }
}  // namespace
