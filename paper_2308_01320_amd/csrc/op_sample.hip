// A token per row of logits from a given random number, after temperature, top-k, top-p and min-p.
#include "operators.h"

namespace he_op {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Order of a row's tokens: larger logits first, of equal ones the lower id.  A token's place in it as one number: a larger place comes first.
__device__ __forceinline__ uint64_t place(float z, int id) {
    const uint32_t u = __float_as_uint(z == 0.f ? 0.f : z);  // (+0 and -0 are equal)
    return ((uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32) | (uint32_t)~id;
}

// Weights exp((z - max) / T) as whole multiples of 2^-42, so that sums do not depend on their order and borders between tokens fall where the
// definition puts them to 2^-43 of the largest weight; 2^20 of them fit 64 bits.
__device__ __forceinline__ uint64_t weight(float z, float top, double rate) {
    if (z == top) return 1ull << 42;
    const double x = ((double)z - (double)top) * rate;  // rate: log2(e) / T
    return x > -44.0 ? (uint64_t)rint(exp2(x + 42.0)) : 0ull;
}

template <class V, class Op>
__device__ __forceinline__ V block_all(V v, V* sh, Op op) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = op(v, sh[w]);
    return v;
}

template <class E>
__global__ __launch_bounds__(kThreads) void sample_kernel(Rows logits, int vocab, Filters f, const float* __restrict__ uniform, int32_t* __restrict__ ids,
                                                          float* __restrict__ logprobs) {
    typedef typename E::T T;
    __shared__ float shf[kWaves];
    __shared__ double shd[kWaves];
    __shared__ unsigned long long shu[kWaves];
    __shared__ unsigned long long upto[kThreads];
    __shared__ int pick;
    const int row = blockIdx.x;
    const T* z = (const T*)logits.data + (int64_t)row * logits.stride;
    auto at = [&](int i) { const float x = E::up(z[i]); return x == x ? x : -INFINITY; };  // a NaN is never drawn
    const auto fmax2 = [](float a, float b) { return fmaxf(a, b); };
    const auto addd = [](double a, double b) { return a + b; };
    const auto addu = [](unsigned long long a, unsigned long long b) { return a + b; };
    float top = -INFINITY;
    for (int i = threadIdx.x; i < vocab; i += kThreads) top = fmaxf(top, at(i));
    top = block_all(top, shf, fmax2);
    if (top == -INFINITY) {
        if (threadIdx.x == 0) {
            ids[row] = -1;
            logprobs[row] = -INFINITY;
        }
        return;
    }
    double lse = 0.0;
    for (int i = threadIdx.x; i < vocab; i += kThreads) {
        const float x = at(i);
        lse += x == top ? 1.0 : exp((double)x - (double)top);
    }
    lse = block_all(lse, shd, addd);
    const float temperature = f.temperature ? f.temperature[row] : 1.f;
    const bool greedy = !(temperature > 0.f);
    const double rate = greedy ? 0.0 : 1.4426950408889634 / (double)temperature;
    const int k = greedy ? 1 : f.top_k ? f.top_k[row] : 0;
    // the last token in order that is kept, as its place
    uint64_t last = 0;
    auto count_from = [&](uint64_t c) {
        unsigned long long n = 0;
        for (int i = threadIdx.x; i < vocab; i += kThreads) n += place(at(i), i) >= c;
        return block_all(n, shu, addu);
    };
    auto mass_from = [&](uint64_t c) {
        unsigned long long n = 0;
        for (int i = threadIdx.x; i < vocab; i += kThreads) {
            const float x = at(i);
            if (place(x, i) >= c) n += weight(x, top, rate);
        }
        return block_all(n, shu, addu);
    };
    if (k > 0 && k < vocab)
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t c = last | (1ull << bit);
            if (count_from(c) >= (unsigned long long)k) last = c;
        }
    const float p = f.top_p && !greedy ? f.top_p[row] : 1.f;
    if (p < 1.f) {
        const double goal = (double)p * (double)mass_from(last);
        uint64_t c0 = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t c = c0 | (1ull << bit);
            if ((double)mass_from(c) >= goal && mass_from(c) > 0) c0 = c;
        }
        last = max(last, c0);
    }
    const float least = f.min_p && !greedy ? f.min_p[row] : 0.f;
    // kept: place >= last, and (z - max) / T >= log(min_p); the largest always
    const double floor_x = least > 0.f ? fmin(log2((double)least), 0.0) : -INFINITY;
    auto kept = [&](float x, int i) {
        return x > -INFINITY && place(x, i) >= last && (x == top || ((double)x - (double)top) * rate >= floor_x);
    };
    // in order of the ids: shares of consecutive ids, their sums added up
    const int each = (vocab + kThreads - 1) / kThreads, i0 = threadIdx.x * each, i1 = min(vocab, i0 + each);
    unsigned long long mine = 0;
    int final = -1;
    for (int i = i0; i < i1; ++i) {
        const float x = at(i);
        const uint64_t w = kept(x, i) ? weight(x, top, rate) : 0;
        mine += w;
        if (w) final = i;
    }
    if (threadIdx.x == 0) pick = -1;
    upto[threadIdx.x] = mine;
    __syncthreads();
    if (final >= 0) atomicMax(&pick, final);
    for (int o = 1; o < kThreads; o <<= 1) {
        const unsigned long long v = (int)threadIdx.x >= o ? upto[threadIdx.x - o] : 0;
        __syncthreads();
        upto[threadIdx.x] += v;
        __syncthreads();
    }
    const unsigned long long total = upto[kThreads - 1], after = upto[threadIdx.x];
    const float u = uniform[row];
    const double goal = u > 0.f ? (double)u * (double)total : 0.0;
    int id = -1;
    if (goal < (double)total) {
        unsigned long long sum = after - mine;
        if ((double)sum <= goal && (double)after > goal)
            for (int i = i0; i < i1; ++i) {
                const float x = at(i);
                if (kept(x, i)) sum += weight(x, top, rate);
                if ((double)sum > goal) { id = i; break; }
            }
    } else if (threadIdx.x == 0) id = pick;  // a number of 1 or more: the last token kept
    if (id >= 0) {
        ids[row] = id;
        const float x = at(id);
        logprobs[row] = (float)((x == top ? 0.0 : (double)x - (double)top) - log(lse));
    }
}

}  // namespace

void sample(hipStream_t s, he_dtype dt, Rows logits, int rows, int vocab, const Filters& f, const float* uniform, int32_t* ids, float* logprobs) {
    by_type(dt, [&](auto e) { sample_kernel<decltype(e)><<<rows, kThreads, 0, s>>>(logits, vocab, f, uniform, ids, logprobs); });
}

}  // namespace he_op
