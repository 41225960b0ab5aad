// Attention of one new token per sequence over a paged cache, split over the cache's length and joined.
#include <algorithm>

#include "bf16_common.h"
#include "op_attend.h"

namespace he_op {
namespace {

// Split `part` of `splits` of a sequence of len positions: equal shares, in whole multiples of 64 positions.
__device__ __forceinline__ void share_of(int len, int splits, int part, int& begin, int& end) {
    const int each = ((len + splits - 1) / splits + 63) & ~63;
    begin = (int)min((int64_t)part * each, (int64_t)len);
    end = min(begin + each, len);
}

// What a split leaves for the join: per (sequence, head, split) maximum and sum, then d weighted values
struct Partial {
    float2* ml;
    float* o;
};
__host__ __device__ inline Partial partial_of(float* workspace, size_t rows, int splits) {
    return {reinterpret_cast<float2*>(workspace), workspace + 2 * rows * splits};
}

template <class E, int DP, int GQ>
__global__ __launch_bounds__(256) void paged_attention_kernel(Cache c, Rows q, int n_heads, Rows out, const int32_t* __restrict__ lens, int splits,
                                                              float scale, float* __restrict__ workspace) {
    typedef typename E::T T;
    __shared__ AttendShared<DP, GQ> sh;
    const int share = n_heads / c.n_kv_heads, groups = (share + GQ - 1) / GQ;
    const int part = blockIdx.x % splits, rest = blockIdx.x / splits, h = rest / groups, g0 = rest % groups * GQ, b = blockIdx.y, d = c.head_dim;
    const int len = (int)min((int64_t)max(lens[b], 0), (int64_t)c.pages_per_seq << c.page_shift);
    int begin, end;
    share_of(len, splits, part, begin, end);
    float qs[GQ][8];
#pragma unroll
    for (int g = 0; g < GQ; ++g)
        query8<E, DP>((const T*)q.data + (int64_t)b * q.stride + (int64_t)(h * share + min(g0 + g, share - 1)) * d, d, scale, qs[g]);
    auto rows = [&](int j, const T*& kp, const T*& vp) {
        const int page = page_of(c, b, j);
        if (page < 0) return false;
        const size_t at = cache_row(c, page, h, j);
        kp = (const T*)c.k + at;
        vp = (const T*)c.v + at;
        return true;
    };
    auto emit = [&](int g, int e, float m, float l, float o) {
        if (g0 + g >= share || e >= d) return;
        const int head = h * share + g0 + g;
        if (splits == 1) {
            const float y = attended(l, o), next = __shfl_xor(y, 1);
            T* op = (T*)out.data + (int64_t)b * out.stride + (int64_t)head * d + e;
            if constexpr (sizeof(T) == 4) *op = y;
            else if (!(e & 1)) *reinterpret_cast<uint32_t*>(op) = E::pack(y, next);
            return;
        }
        const size_t row = ((size_t)b * n_heads + head) * splits + part;
        const Partial p = partial_of(workspace, (size_t)gridDim.y * n_heads, splits);
        if (e == 0) p.ml[row] = make_float2(m, l);
        p.o[row * d + e] = o;
    };
    attend<E, DP, GQ>(sh, begin, end, d, qs, rows, emit);
}

// The splits of a row, weighted by exp(their maximum - the largest)
template <class E>
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ workspace, Rows out, int n_heads, int d, int splits) {
    typedef typename E::T T;
    const int row = blockIdx.x, b = row / n_heads, h = row % n_heads, e = threadIdx.x;
    const Partial p = partial_of(const_cast<float*>(workspace), gridDim.x, splits);
    float top = -INFINITY;
    for (int s = 0; s < splits; ++s) top = fmaxf(top, p.ml[(size_t)row * splits + s].x);
    float l = 0.f, o = 0.f;
    for (int s = 0; s < splits; ++s) {
        const float2 a = p.ml[(size_t)row * splits + s];
        if (a.y == 0.f) continue;  // a split that saw no key
        const float f = a.x > -INFINITY ? expf(a.x - top) : a.y;
        l += a.y * f;
        if (e < d) o += p.o[((size_t)row * splits + s) * d + e] * f;
    }
    if (e >= d) return;
    const float y = attended(l, o), next = __shfl_xor(y, 1);
    T* op = (T*)out.data + (int64_t)b * out.stride + (int64_t)h * d + e;
    if constexpr (sizeof(T) == 4) *op = y;
    else if (!(e & 1)) *reinterpret_cast<uint32_t*>(op) = E::pack(y, next);
}

}  // namespace

int paged_splits(he_dtype dt, int n_heads, int n_kv_heads, int head_dim, int n_seqs, int max_len) {
    const int64_t groups = (int64_t)n_seqs * n_kv_heads;
    const int64_t want = std::max<int64_t>(1, 4 * he_bf16::num_cus() / std::max<int64_t>(1, groups));
    return (int)std::min<int64_t>(std::min<int64_t>(want, 64), std::max(1, (max_len + 127) / 128));
}

void paged_attention(hipStream_t s, he_dtype dt, const Cache& c, Rows q, int n_heads, Rows out, const int32_t* lens, int n_seqs, int splits,
                     float scale, float* workspace) {
    const int share = n_heads / c.n_kv_heads;
    by_type(dt, [&](auto e) {
        typedef decltype(e) E;
        auto launch = [&](auto dp, auto gq) {
            constexpr int DP = decltype(dp)::value, GQ = decltype(gq)::value;
            const int groups = (share + GQ - 1) / GQ;
            paged_attention_kernel<E, DP, GQ><<<dim3(c.n_kv_heads * groups * splits, n_seqs), 256, 0, s>>>(c, q, n_heads, out, lens, splits, scale, workspace);
        };
        auto by_heads = [&](auto dp) {
            if (share == 1) launch(dp, std::integral_constant<int, 1>{});
            else if (share == 2) launch(dp, std::integral_constant<int, 2>{});
            else launch(dp, std::integral_constant<int, 4>{});
        };
        if (c.head_dim <= 64) by_heads(std::integral_constant<int, 64>{});
        else if (c.head_dim <= 128) by_heads(std::integral_constant<int, 128>{});
        else by_heads(std::integral_constant<int, 256>{});
        if (splits > 1) join_kernel<E><<<n_seqs * n_heads, 256, 0, s>>>(workspace, out, n_heads, c.head_dim, splits);
    });
}

}  // namespace he_op
