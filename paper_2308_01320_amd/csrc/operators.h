// Shared by the operators that stand beside the engine (include/he.h: he_paged_append, he_paged_attention, he_packed_attention,
// he_sample): element types, rows of tokens, the paged cache as kernels see it, and the launchers.
#pragma once
#include "../../include/he.h"
#include "he_common.h"

namespace he_op {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Element types.  A lane's unit of work is eight values of a row: 16 bytes of the 16-bit types, 32 of float.
struct F32 {
    typedef float T;
    static __device__ __forceinline__ float up(float v) { return v; }
};
struct BF16 {
    typedef uint16_t T;
    static __device__ __forceinline__ float up(uint16_t v) { return bf16_to_f32(v); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return f32x2_to_bf16x2(lo, hi); }
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
};
struct F16 {
    typedef uint16_t T;
    static __device__ __forceinline__ float up(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        typedef float v2f __attribute__((ext_vector_type(2)));
        typedef _Float16 v2h __attribute__((ext_vector_type(2)));
        const v2f v = {lo, hi};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, v2h));
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w & 0xFFFFu)); }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16)); }
};

// Eight values as they lie in memory (16-byte aligned)
template <class E> struct Raw8 { u32x4 w; };
template <> struct Raw8<F32> { float4 a, b; };

template <class E> __device__ __forceinline__ Raw8<E> zero8() { return Raw8<E>{u32x4{0u, 0u, 0u, 0u}}; }
template <> __device__ __forceinline__ Raw8<F32> zero8<F32>() { return Raw8<F32>{make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)}; }
template <class E> __device__ __forceinline__ Raw8<E> load8(const typename E::T* p) { return *reinterpret_cast<const Raw8<E>*>(p); }
template <class E> __device__ __forceinline__ void store8(typename E::T* p, const Raw8<E>& r) { *reinterpret_cast<Raw8<E>*>(p) = r; }

template <class E> __device__ __forceinline__ void unpack8(const Raw8<E>& r, float (&f)[8]) {
    f[0] = E::lo(r.w.x); f[1] = E::hi(r.w.x); f[2] = E::lo(r.w.y); f[3] = E::hi(r.w.y);
    f[4] = E::lo(r.w.z); f[5] = E::hi(r.w.z); f[6] = E::lo(r.w.w); f[7] = E::hi(r.w.w);
}
template <> __device__ __forceinline__ void unpack8<F32>(const Raw8<F32>& r, float (&f)[8]) {
    f[0] = r.a.x; f[1] = r.a.y; f[2] = r.a.z; f[3] = r.a.w; f[4] = r.b.x; f[5] = r.b.y; f[6] = r.b.z; f[7] = r.b.w;
}
template <class E> __device__ __forceinline__ Raw8<E> pack8(const float (&f)[8]) {
    return Raw8<E>{u32x4{E::pack(f[0], f[1]), E::pack(f[2], f[3]), E::pack(f[4], f[5]), E::pack(f[6], f[7])}};
}
template <> __device__ __forceinline__ Raw8<F32> pack8<F32>(const float (&f)[8]) {
    return Raw8<F32>{make_float4(f[0], f[1], f[2], f[3]), make_float4(f[4], f[5], f[6], f[7])};
}

// One instance of f per element type
template <class Fn>
inline void by_type(he_dtype t, Fn f) {
    if (t == HE_F32) f(F32{});
    else if (t == HE_BF16) f(BF16{});
    else f(F16{});
}

// Rows of a packed batch: row i starts at data + i * stride, its heads lie side by side
struct Rows { void* data; int64_t stride; };

// The cache as a kernel sees it.  page_shift: log2 of the positions to a page
struct Cache {
    void *k, *v;
    const int32_t* pages;
    int n_pages, pages_per_seq, page_shift, n_kv_heads, head_dim;
    int64_t page_stride;
};
// The page that holds position t >= 0 of sequence b, or -1: the table has no such entry, or the entry names no page
__device__ __forceinline__ int page_of(const Cache& c, int b, int t) {
    const int i = t >> c.page_shift;
    if (i >= c.pages_per_seq) return -1;
    const int p = c.pages[(size_t)b * c.pages_per_seq + i];
    return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}
// Where position t of key-value head h begins in page p, in elements from the start of K (or V)
__device__ __forceinline__ size_t cache_row(const Cache& c, int p, int h, int t) {
    return (size_t)p * c.page_stride + (((size_t)h << c.page_shift) + (t & ((1 << c.page_shift) - 1))) * c.head_dim;
}

// The sequence that packed row i belongs to: the last b of [0, n) with starts[b] <= i.  Sixty-four probes a step (one for each lane),
// so two dependent loads reach 4096 sequences.  Ends, and stays inside the table, whatever the table holds.
__device__ __forceinline__ int seq_of_row(const int32_t* starts, int n, int i) {
    const int lane = threadIdx.x & 63;
    int lo = 0, span = n;
    while (span > 1) {
        const int step = (span + 63) / 64, at = lane * step;
        const int below = __popcll(__ballot(at < span && starts[lo + at] <= i));
        const int k = max(below, 1) - 1;
        lo += k * step;
        span = min(step, span - k * step);
    }
    return lo;
}

// ---- launchers
struct Rope { int half, interleaved; double turns[128]; };  // half the rotated dimensions; turns a position adds to pair i
void append(hipStream_t s, he_dtype dt, const Cache& c, const Rope& rope, Rows q, int n_heads, Rows q_out, Rows k, Rows k_out, Rows v,
            const int32_t* starts, const int32_t* lens, int n_seqs, int n_tokens);

int paged_splits(he_dtype dt, int page_size, int n_heads, int n_kv_heads, int n_seqs, int max_len);
void paged_attention(hipStream_t s, he_dtype dt, const Cache& c, Rows q, int n_heads, Rows out, const int32_t* lens, int n_seqs, int splits,
                     float scale, float* workspace);

void packed_attention(hipStream_t s, he_dtype dt, Rows q, int n_heads, Rows k, Rows v, int n_kv_heads, int head_dim, Rows out,
                      const int32_t* starts, int n_seqs, int n_tokens, bool causal, float scale);

struct Filters { const float* temperature; const int32_t* top_k; const float *top_p, *min_p; };
size_t sample_workspace(int rows, int vocab);
void sample(hipStream_t s, he_dtype dt, Rows logits, int rows, int vocab, const Filters& f, const float* uniform, int32_t* ids, float* logprobs,
            void* workspace);

}  // namespace he_op
