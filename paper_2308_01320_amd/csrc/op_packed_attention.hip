// Attention over whole prompts laid end to end.
#include <algorithm>

#include "bf16_common.h"
#include "op_attend.h"

namespace he_op {
namespace {

template <class E, int DP>
__global__ __launch_bounds__(256) void packed_attention_kernel(Rows q, int n_heads, Rows k, Rows v, int n_kv_heads, int d, Rows out,
                                                               const int32_t* __restrict__ starts, int n_seqs, int n_tokens, int causal, float scale) {
    typedef typename E::T T;
    __shared__ AttendShared<DP, 1> sh;
    const int h = blockIdx.x, i = blockIdx.y + 32768 * blockIdx.z, hk = h / (n_heads / n_kv_heads);
    if (i >= n_tokens || i < starts[0] || i >= starts[n_seqs]) return;
    const int b = seq_of_row(starts, n_seqs, i);
    const int begin = max(starts[b], 0), end = min(causal ? i + 1 : starts[b + 1], n_tokens);
    float qs[1][8];
    query8<E, DP>((const T*)q.data + (int64_t)i * q.stride + (int64_t)h * d, d, scale, qs[0]);
    auto rows = [&](int j, const T*& kp, const T*& vp) {
        kp = (const T*)k.data + (int64_t)j * k.stride + (int64_t)hk * d;
        vp = (const T*)v.data + (int64_t)j * v.stride + (int64_t)hk * d;
        return true;
    };
    auto emit = [&](int, int e, float, float l, float o) {
        if (e >= d) return;
        const float y = attended(l, o), next = __shfl_xor(y, 1);
        T* op = (T*)out.data + (int64_t)i * out.stride + (int64_t)h * d + e;
        if constexpr (sizeof(T) == 4) *op = y;
        else if (!(e & 1)) *reinterpret_cast<uint32_t*>(op) = E::pack(y, next);
    };
    attend<E, DP, 1>(sh, begin, end, d, qs, rows, emit);
}

}  // namespace

void packed_attention(hipStream_t s, he_dtype dt, Rows q, int n_heads, Rows k, Rows v, int n_kv_heads, int head_dim, Rows out,
                      const int32_t* starts, int n_seqs, int n_tokens, bool causal, float scale) {
    by_type(dt, [&](auto e) {
        typedef decltype(e) E;
        const dim3 grid(n_heads, std::min(n_tokens, 32768), (n_tokens + 32767) / 32768);
        auto launch = [&](auto dp) {
            packed_attention_kernel<E, decltype(dp)::value><<<grid, 256, 0, s>>>(q, n_heads, k, v, n_kv_heads, head_dim, out, starts, n_seqs, n_tokens, causal, scale);
        };
        if (head_dim <= 64) launch(std::integral_constant<int, 64>{});
        else if (head_dim <= 128) launch(std::integral_constant<int, 128>{});
        else launch(std::integral_constant<int, 256>{});
    });
}

}  // namespace he_op
