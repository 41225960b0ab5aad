// New keys and values into a paged cache, with queries and keys rotated by their positions on the way.
#include "operators.h"

namespace he_op {
namespace {

// y = x turned: pair i = (x_i, x_{i + r/2}), or (x_2i, x_{2i+1}) with `interleaved`, of the first r dimensions by the angle
// position * scale * base^(-2 i / r); the rest of the row as it is.
//
// A position may be in the hundred thousands, where a float angle is off by hundredths: the turns (angle / 2 pi) are a product in 64 bits
// of which only the fraction is kept, and sine and cosine are taken of that in float (2^-26 of a turn).  The rotation is float, rounded
// once to the row's type.
//
// A workgroup takes a token: its first r/2 threads leave the sines and cosines in LDS, then a thread takes sixteen values of a head --
// the two groups of eight that are each other's pairs, or eight pairs -- and goes over the heads of queries, keys and values 256 / (d/16)
// apart, always with the same pairs, whose sines stay in registers.  Bound by memory: 8192 rows at most of 120 heads of 128 (321 MB) take 70 us, 4.6 TB/s
// where a plain copy of 2 GiB reaches 5.1; a step of 32 rows of 56 heads 3.5 us in a graph, a launch and three dependent loads.  The values of the
// first heads requested ahead of the position: 72.7 us for 70.8 and 7.0 for 5.0 (kernel times by themselves), more registers and no less waiting.
template <class E>
__global__ __launch_bounds__(256) void append_kernel(Cache c, Rope rope, Rows q, int n_heads, Rows q_out, Rows k, Rows k_out, Rows v,
                                                     const int32_t* __restrict__ starts, const int32_t* __restrict__ lens, int n_seqs) {
    typedef typename E::T T;
    __shared__ __align__(16) float cs[2][128];
    const int i = blockIdx.x, d = c.head_dim;
    int b = i, first = i;
    if (starts) {
        if (i < starts[0] || i >= starts[n_seqs]) return;  // a row of no sequence
        b = seq_of_row(starts, n_seqs, i);
        first = starts[b];
    }
    const int pos = lens[b] + (i - first);
    const int page = pos >= 0 ? page_of(c, b, pos) : -1;
    if ((int)threadIdx.x < rope.half) {
        const double turns = (double)pos * rope.turns[threadIdx.x];
        float sn, cn;
        sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cn);
        cs[0][threadIdx.x] = cn;
        cs[1][threadIdx.x] = sn;
    }
    __syncthreads();
    const int units = d >> 4, u = threadIdx.x % units, slots = 256 / units, slot = threadIdx.x / units;
    if (slot >= slots) return;
    // where this thread's two groups of eight begin, and its pairs' cosines and sines
    const bool turned = u < (rope.half >> 3), apart = turned && !rope.interleaved;
    const int e0 = apart ? u * 8 : u * 16, e1 = apart ? u * 8 + rope.half : u * 16 + 8;  // (rope.half is a multiple of 8)
    const int f0 = u * 16, f1 = u * 16 + 8;                                              // values are not turned
    float cn[8], sn[8];
    if (turned) {
#pragma unroll
        for (int x = 0; x < 8; ++x) { cn[x] = cs[0][u * 8 + x]; sn[x] = cs[1][u * 8 + x]; }
    }
    const int nq = q.data ? n_heads : 0, total = nq + 2 * c.n_kv_heads;
    for (int hh = blockIdx.y * slots + slot; hh < total; hh += gridDim.y * slots) {
        const bool is_q = hh < nq, is_v = hh >= nq + c.n_kv_heads;
        const int h = is_q ? hh : is_v ? hh - nq - c.n_kv_heads : hh - nq;
        const Rows& src = is_q ? q : is_v ? v : k;
        const T* p = (const T*)src.data + (int64_t)i * src.stride + (int64_t)h * d;
        const int o0 = is_v ? f0 : e0, o1 = is_v ? f1 : e1;
        Raw8<E> r0 = load8<E>(p + o0), r1 = load8<E>(p + o1);
        if (turned && !is_v) {
            float a[8], z[8];
            unpack8<E>(r0, a);
            unpack8<E>(r1, z);
            if (rope.interleaved) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float a0 = a[2 * x], a1 = a[2 * x + 1], z0 = z[2 * x], z1 = z[2 * x + 1];
                    a[2 * x] = a0 * cn[x] - a1 * sn[x];
                    a[2 * x + 1] = a0 * sn[x] + a1 * cn[x];
                    z[2 * x] = z0 * cn[4 + x] - z1 * sn[4 + x];
                    z[2 * x + 1] = z0 * sn[4 + x] + z1 * cn[4 + x];
                }
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const float a0 = a[x], z0 = z[x];
                    a[x] = a0 * cn[x] - z0 * sn[x];
                    z[x] = a0 * sn[x] + z0 * cn[x];
                }
            }
            r0 = pack8<E>(a);
            r1 = pack8<E>(z);
        }
        if (is_q) {
            T* o = (T*)q_out.data + (int64_t)i * q_out.stride + (int64_t)h * d;
            store8<E>(o + o0, r0);
            store8<E>(o + o1, r1);
            continue;
        }
        if (!is_v && k_out.data) {
            T* o = (T*)k_out.data + (int64_t)i * k_out.stride + (int64_t)h * d;
            store8<E>(o + o0, r0);
            store8<E>(o + o1, r1);
        }
        if (page >= 0) {
            T* o = (T*)(is_v ? c.v : c.k) + cache_row(c, page, h, pos);
            store8<E>(o + o0, r0);
            store8<E>(o + o1, r1);
        }
    }
}

}  // namespace

void append(hipStream_t s, he_dtype dt, const Cache& c, const Rope& rope, Rows q, int n_heads, Rows q_out, Rows k, Rows k_out, Rows v,
            const int32_t* starts, const int32_t* lens, int n_seqs, int n_tokens) {
    by_type(dt, [&](auto e) {
        append_kernel<decltype(e)><<<dim3(n_tokens, 1), 256, 0, s>>>(c, rope, q, n_heads, q_out, k, k_out, v, starts, lens, n_seqs);
    });
}

}  // namespace he_op
