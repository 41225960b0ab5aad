// A token per row of logits from a given random number, after temperature, top-k, top-p and min-p.
//
// Tokens are ordered by (logit descending, id ascending), and each filter keeps a first part of that order; the number then picks from the kept
// weights w = exp((z - max z) / T) in order of the ids.  Which token that is hangs on sums of up to 2^20 weights against borders between
// two of them, so weights are whole multiples of 2^-42 computed to 1e-11 of themselves (weight()) and summed as 64-bit integers: no order of
// summation, not even that of the LDS atomics, changes an id.
//
// One workgroup of sixteen wavefronts takes a row and goes over it a few times (it comes out of the L2 after the first): the maximum; then the sum of
// the soft-max and, for top-k and top-p, a histogram of counts and weights over 2753 steps of 1/64 in log2 w, whose running sums name the
// step in which a filter's border lies; the tokens of that step alone, each counting who comes before it; then the kept weights, a
// contiguous span of ids to each wavefront; and the wavefront in whose span the number falls goes over it once more.
#include <climits>

#include "operators.h"

namespace he_op {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kUnit = 42 * 1024;                // log2 of the largest weight, in 1024ths: weights are in units of 2^-42
constexpr int kBins = (kUnit + 1024) / 16 + 1;  // steps of 16 / 1024 in log2, down to a weight of half a unit
constexpr int kList = 2048;                     // tokens of a step that are compared one with another

// A token's place in the order as one number: a larger place comes first.
__device__ __forceinline__ uint64_t place(float z, int id) {
    const uint32_t u = __float_as_uint(z == 0.f ? 0.f : z);  // (+0 and -0 are equal)
    return ((uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32) | (uint32_t)~id;
}
__device__ __forceinline__ float place_logit(uint64_t p) {
    const uint32_t u = (uint32_t)(p >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}

struct Shared {
    double pow2[1024];                  // 2^(j / 1024)
    unsigned long long mass[kBins];
    unsigned int count[kBins];
    unsigned long long list_place[kList], list_weight[kList];
    unsigned long long wave_u[kWaves], wave_u2[kWaves];
    double wave_d[kWaves];
    float wave_f[kWaves];
    int bin, list_n, id;
    unsigned long long before_count, before_mass, last, kept_mass;
};

// (z - max) log2(e) / T + 42 in 1024ths: what of it is whole (`log`) and what is left of it, up to half a 1024th.  Zero: less than half a unit
// of weight, or nothing at all.
struct Log { int whole; float rest; bool zero; };
__device__ __forceinline__ Log log_weight(float z, double top, double rate) {
    constexpr double kRound = 6755399441055744.0;  // 1.5 2^52: adding it rounds to whole numbers, which are then its low bits
    const double u = fma((double)z - top, rate, (double)kUnit), m = u + kRound;
    return {(int)(uint32_t)__double_as_longlong(m), (float)(u - (m - kRound)), !(u >= -1024.0)};
}
// 2^((whole + rest) / 1024) to the nearest whole number: a table for the whole part, and for the rest a polynomial in float, whose 2^-24 is of a
// correction of 2^-11.4 at most (the cubic term left out is 7e-12).
__device__ __forceinline__ unsigned long long weight(const Log& l, const double* pow2) {
    constexpr float c = 6.769015435155716e-4f;  // ln 2 / 1024
    const float q = l.rest * fmaf(l.rest, 0.5f * c * c, c);
    const double t = pow2[l.whole & 1023], w = fma(t, (double)q, t);
    const double scaled = __longlong_as_double(__double_as_longlong(w) + ((long long)(l.whole >> 10) << 52));
    return l.zero ? 0ull : (unsigned long long)__double_as_longlong(scaled + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;  // + 2^52
}

template <class V, class Op>
__device__ __forceinline__ V wave_all(V v, Op op) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o));
    return v;
}
template <class V, class Op>
__device__ __forceinline__ V block_all(V v, V* sh, Op op) {
    v = wave_all(v, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = op(v, sh[w]);
    return v;
}
// sums of v over the lanes up to and including this one
__device__ __forceinline__ unsigned long long wave_upto(unsigned long long v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long x = __shfl_up(v, o);
        if (lane >= o) v += x;
    }
    return v;
}

// A row as the sixteen wavefronts take it: 16 bytes to a lane, spans of consecutive ids to a wavefront.  Pieces lie on 16 bytes whatever the row
// does; those that are not wholly inside it are read value by value.
template <class E>
struct Row {
    typedef typename E::T T;
    static constexpr int N = 16 / sizeof(T);
    const T* z;
    int vocab, off, per_wave, pieces;
    bool infinite;  // the largest logit is +infinity: such tokens weigh the same, the others nothing
    __device__ __forceinline__ Row(const T* p, int v) : z(p), vocab(v), infinite(false) {
        off = (int)(((uintptr_t)p & 15) / sizeof(T));
        pieces = (vocab + off + N - 1) / N;
        per_wave = ((pieces + kWaves - 1) / kWaves + 63) & ~63;
    }
    __device__ __forceinline__ int first(int piece) const { return piece * N - off; }
    __device__ __forceinline__ void load(int piece, float (&x)[N]) const {
        const int i0 = first(piece);
        if (i0 >= 0 && i0 + N <= vocab) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(z + i0);
            if constexpr (N == 4) {
                x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
            } else {
                x[0] = E::lo(w.x); x[1] = E::hi(w.x); x[2] = E::lo(w.y); x[3] = E::hi(w.y);
                x[4] = E::lo(w.z); x[5] = E::hi(w.z); x[6] = E::lo(w.w); x[7] = E::hi(w.w);
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = i0 + e >= 0 && i0 + e < vocab ? E::up(z[i0 + e]) : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = fmaxf(x[e], -INFINITY);  // a NaN is never drawn
        if (infinite) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = x[e] == INFINITY ? 0.f : -INFINITY;
        }
    }
    // f(first id, values) for every piece of this lane, in order of the ids along a lane and across the lanes of a round
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        const int wave = threadIdx.x >> 6, end = min(pieces, (wave + 1) * per_wave);
        for (int piece = wave * per_wave + (threadIdx.x & 63); piece < end; piece += 64) {
            float x[N];
            load(piece, x);
            f(first(piece), x);
        }
    }
};

// The place of the last token kept, of a filter whose border lies in step `bin`: before it `before` tokens' count (or weight) comes from larger
// steps, and the border is the first token at which it reaches `goal`.  Also leaves the weight up to and including that token in sh.kept_mass.
template <class E>
__device__ uint64_t border(Shared& sh, const Row<E>& row, double top, double rate, int bin, bool by_count, unsigned long long before_count,
                           unsigned long long before_mass, double goal) {
    constexpr int N = Row<E>::N;
    __syncthreads();
    if (threadIdx.x == 0) sh.list_n = 0;
    __syncthreads();
    row.each([&](int i0, const float (&x)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const Log l = log_weight(x[e], top, rate);
            if (!l.zero && (kUnit - l.whole) >> 4 == bin) {
                const int at = atomicAdd(&sh.list_n, 1);
                if (at < kList) {
                    sh.list_place[at] = place(x[e], i0 + e);
                    sh.list_weight[at] = weight(l, sh.pow2);
                }
            }
        }
    });
    __syncthreads();
    const int n = sh.list_n;
    if (n <= kList) {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const unsigned long long mine = sh.list_place[i];
            unsigned long long count = before_count, mass = before_mass;
            for (int j = 0; j < n; ++j)
                if (sh.list_place[j] > mine) {
                    ++count;
                    mass += sh.list_weight[j];
                }
            const unsigned long long w = sh.list_weight[i];
            if (by_count ? (double)count < goal && (double)(count + 1) >= goal : (double)mass < goal && (double)(mass + w) >= goal) {
                sh.last = mine;
                sh.kept_mass = mass + w;
            }
        }
        __syncthreads();
        return sh.last;
    }
    // A step with thousands of tokens in it (a flat row, or one of few different values): the border's place bit by bit, from the first in which
    // the step's places differ.
    const auto addu = [](unsigned long long a, unsigned long long b) { return a + b; };
    auto of_bin = [&](auto f) {
        row.each([&](int i0, const float (&x)[N]) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const Log l = log_weight(x[e], top, rate);
                if (!l.zero && (kUnit - l.whole) >> 4 == bin) f(place(x[e], i0 + e), l);
            }
        });
    };
    unsigned long long ones = ~0ull, any = 0;
    of_bin([&](uint64_t p, const Log&) { ones &= p; any |= p; });
    ones = block_all(ones, sh.wave_u, [](unsigned long long a, unsigned long long b) { return a & b; });
    any = block_all(any, sh.wave_u, [](unsigned long long a, unsigned long long b) { return a | b; });
    const int bits = 64 - __clzll((long long)(ones ^ any));  // (they differ: ids do)
    unsigned long long last = bits == 64 ? 0ull : ones >> bits << bits;
    auto from = [&](unsigned long long c, unsigned long long& count, unsigned long long& mass) {
        count = before_count;
        mass = before_mass;
        unsigned long long n_mine = 0, m_mine = 0;
        of_bin([&](uint64_t p, const Log& l) { if (p >= c) { ++n_mine; m_mine += weight(l, sh.pow2); } });
        count += block_all(n_mine, sh.wave_u, addu);
        mass += block_all(m_mine, sh.wave_u, addu);
    };
    unsigned long long count, mass;
    for (int b = bits - 1; b >= 0; --b) {
        const unsigned long long c = last | 1ull << b;
        from(c, count, mass);
        if (by_count ? (double)count >= goal : (double)mass >= goal) last = c;
    }
    from(last, count, mass);
    if (threadIdx.x == 0) sh.kept_mass = mass;
    __syncthreads();
    return last;
}

template <class E>
__global__ __launch_bounds__(kThreads) void sample_kernel(Rows logits, int vocab, Filters f, const float* __restrict__ uniform, int32_t* __restrict__ ids,
                                                          float* __restrict__ logprobs) {
    typedef typename E::T T;
    constexpr int N = Row<E>::N;
    __shared__ Shared sh;
    const int r = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Row<E> row((const T*)logits.data + (int64_t)r * logits.stride, vocab);
    const auto addu = [](unsigned long long a, unsigned long long b) { return a + b; };

    float best = -INFINITY;
    row.each([&](int, const float (&x)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) best = fmaxf(best, x[e]);
    });
    const float temperature = f.temperature ? f.temperature[r] : 1.f, u = uniform[r];
    int k = f.top_k ? f.top_k[r] : 0;
    const float p = f.top_p ? f.top_p[r] : 1.f, least = f.min_p ? f.min_p[r] : 0.f;
    sh.pow2[threadIdx.x] = exp2((double)threadIdx.x / 1024.0);
    for (int i = threadIdx.x; i < kBins; i += kThreads) { sh.mass[i] = 0; sh.count[i] = 0; }
    if (threadIdx.x == 0) sh.id = INT_MAX;
    best = block_all(best, sh.wave_f, [](float a, float b) { return fmaxf(a, b); });
    if (best == -INFINITY) {
        if (threadIdx.x == 0) {
            ids[r] = -1;
            logprobs[r] = -INFINITY;
        }
        return;
    }
    row.infinite = best == INFINITY;
    const float topf = row.infinite ? 0.f : best;
    const double top = topf;
    if (!(temperature > 0.f) || p <= 0.f || least > 1.f) k = 1;  // the first in order alone
    const bool first_only = k == 1, top_k = k > 1 && k < vocab, top_p = p < 1.f && !first_only;
    const double rate = first_only ? 0.0 : 1024.0 * 1.4426950408889634 / (double)temperature;

    // the soft-max's sum (in float but for the additions: 2^-24 of each term, in no one direction), with it the histogram, or the first id of the largest
    auto soft = [&](float x) {
        const float d = x - topf;
        return (double)__builtin_amdgcn_exp2f(fmaf(d, 1.44269502f, d * 1.92596299e-8f));  // log2 e in two parts
    };
    double lse = 0.0;
    unsigned long long total = 0;
    if (first_only) {
        int id = INT_MAX;
        row.each([&](int i0, const float (&x)[N]) {
#pragma unroll
            for (int e = N - 1; e >= 0; --e) {
                lse += soft(x[e]);
                if (x[e] == topf) id = min(id, i0 + e);
            }
        });
        if (id != INT_MAX) atomicMin(&sh.id, id);
        lse = block_all(lse, sh.wave_d, [](double a, double b) { return a + b; });
        if (threadIdx.x == 0) {
            ids[r] = sh.id;
            logprobs[r] = (float)-log(lse);
        }
        return;
    }
    // kept: logits above `limit`, and equal to it up to id `limit_id`
    float limit = -INFINITY;
    int limit_id = INT_MAX;
    if (top_k || top_p) {
        row.each([&](int, const float (&x)[N]) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                lse += soft(x[e]);
                const Log l = log_weight(x[e], top, rate);
                if (l.zero) continue;
                const int bin = (kUnit - l.whole) >> 4;
                atomicAdd(&sh.mass[bin], weight(l, sh.pow2));
                if (top_k) atomicAdd(&sh.count[bin], 1u);
            }
        });
        __syncthreads();
        // running sums over the steps, three to a thread
        constexpr int PER = (kBins + kThreads - 1) / kThreads;
        unsigned long long c[PER], m[PER], cs = 0, ms = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = threadIdx.x * PER + i;
            c[i] = at < kBins ? sh.count[at] : 0;
            m[i] = at < kBins ? sh.mass[at] : 0;
            cs += c[i];
            ms += m[i];
        }
        unsigned long long cu = wave_upto(cs), mu = wave_upto(ms);
        if (lane == 63) { sh.wave_u[wave] = cu; sh.wave_u2[wave] = mu; }
        __syncthreads();
        unsigned long long c_all = 0, m_all = 0;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) { cu += sh.wave_u[w]; mu += sh.wave_u2[w]; }
            c_all += sh.wave_u[w];
            m_all += sh.wave_u2[w];
        }
        cu -= cs;  // before this thread's steps
        mu -= ms;
        uint64_t last = 0;
        auto find = [&](bool by_count, double goal) {
            unsigned long long cb = cu, mb = mu;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const unsigned long long b = by_count ? cb : mb, a = by_count ? cb + c[i] : mb + m[i];
                if ((double)b < goal && (double)a >= goal) { sh.bin = threadIdx.x * PER + i; sh.before_count = cb; sh.before_mass = mb; }
                cb += c[i];
                mb += m[i];
            }
            __syncthreads();
            return border(sh, row, top, rate, sh.bin, by_count, sh.before_count, sh.before_mass, goal);
        };
        unsigned long long of_first = m_all;  // weight of the first k
        if (top_k && c_all > (unsigned long long)k) {
            last = find(true, (double)k);
            of_first = sh.kept_mass;
            __syncthreads();
        }
        if (top_p) {
            const uint64_t at = find(false, (double)p * (double)of_first);
            last = at > last ? at : last;
        }
        if (last) {
            limit = place_logit(last);
            limit_id = (int)~(uint32_t)last;
        }
    }
    if (least > 0.f) {
        // w >= min_p as a bound on the logit, up to the next float
        const double bound = top + log2((double)least) * 1024.0 / rate;
        float b = (float)bound;
        if ((double)b < bound) b = nextafterf(b, INFINITY);
        if (b > limit) { limit = fminf(b, topf); limit_id = INT_MAX; }
    }
    const bool summed = top_k || top_p;
    auto kept = [&](float x, int i) { return x > limit || (x == limit && i <= limit_id); };
    unsigned long long mine = 0;
    int final = -1;
    row.each([&](int i0, const float (&x)[N]) {
        if (!summed) {
#pragma unroll
            for (int e = 0; e < N; ++e) lse += soft(x[e]);
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (kept(x[e], i0 + e)) {
                const unsigned long long w = weight(log_weight(x[e], top, rate), sh.pow2);
                mine += w;
                if (w) final = i0 + e;
            }
    });
    lse = block_all(lse, sh.wave_d, [](double a, double b) { return a + b; });
    const unsigned long long of_wave = wave_all(mine, addu);
    const int last_id = wave_all(final, [](int a, int b) { return max(a, b); });
    if (lane == 0) { sh.wave_u[wave] = of_wave; sh.list_place[wave] = (unsigned long long)(uint32_t)(last_id + 1); }
    __syncthreads();
    unsigned long long before = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sh.wave_u[w];
        total += sh.wave_u[w];
    }
    const double goal = u > 0.f ? (double)u * (double)total : 0.0;
    float logit = 0.f;
    int id = -1;
    if (!(goal < (double)total)) {  // a number of 1 or more: the last token kept
        if (threadIdx.x == 0) {
            int most = 0;
            for (int w = 0; w < kWaves; ++w) most = max(most, (int)sh.list_place[w]);
            id = most - 1;
        }
    } else if ((double)before <= goal && (double)(before + of_wave) > goal) {  // (one wavefront)
        const int end = min(row.pieces, (wave + 1) * row.per_wave);
        for (int p0 = wave * row.per_wave; p0 < end; p0 += 64) {
            float x[N];
            unsigned long long w[N], sum = 0;
            const int piece = min(p0 + lane, end - 1), i0 = row.first(piece);
            row.load(piece, x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                w[e] = p0 + lane < end && kept(x[e], i0 + e) ? weight(log_weight(x[e], top, rate), sh.pow2) : 0ull;
                sum += w[e];
            }
            const unsigned long long upto = before + wave_upto(sum);
            if ((double)(upto - sum) <= goal && (double)upto > goal) {  // (one lane)
                unsigned long long s = upto - sum;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    s += w[e];
                    if (id < 0 && (double)s > goal) id = i0 + e;
                }
            }
            if (__any(id >= 0)) break;
            before = __shfl(upto, 63);
        }
    }
    if (id >= 0) {
        logit = fmaxf(E::up(row.z[id]), -INFINITY);
        ids[r] = id;
        logprobs[r] = (float)((row.infinite ? 0.0 : (double)logit - top) - log(lse));
    }
}

}  // namespace

void sample(hipStream_t s, he_dtype dt, Rows logits, int rows, int vocab, const Filters& f, const float* uniform, int32_t* ids, float* logprobs) {
    by_type(dt, [&](auto e) { sample_kernel<decltype(e)><<<rows, kThreads, 0, s>>>(logits, vocab, f, uniform, ids, logprobs); });
}

}  // namespace he_op
