// A token per row of logits from a given random number, after temperature, top-k, top-p and min-p.
//
// Tokens are ordered by (logit descending, id ascending), and each filter keeps a first part of that order; the number then picks from the kept
// weights w = exp((z - max z) / T) in order of the ids.  Which token that is hangs on sums of up to 2^20 weights against borders between
// two of them, so weights are whole multiples of 2^-42 computed to 1e-11 of themselves (weight()) and summed as 64-bit integers: no order of
// summation, not even that of the LDS atomics, changes an id.
//
// Two launches.  slice_kernel goes over the logits once, 4096 ids to a workgroup and sixteen values to a thread's registers: the slice's maximum,
// its head -- the logits from its `cut` up, some seven hundred -- and what the others weigh in the soft-max and at the row's temperature (or,
// for a row without filters, what all of them weigh).  sample_kernel takes a row, the heads of its slices into LDS.  If the filters keep
// nothing below the highest cut, which is the rule, those are all there is from there on: a histogram of counts and weights over steps of
// log2 w names the step in which a filter's border lies, the tokens of that step are compared one with another, and the kept weights are
// summed by spans of ids.  A row without filters needs one slice again, the one in which the number falls.  Else (flat rows) the same is done
// over the whole row, with its own weights.
//
// What bounds it: 64-bit arithmetic (a weight is some 35 instructions, a third of them on doubles) and, in a row's one workgroup, the barriers and
// passes one behind the other.  256 rows of 50272 bf16 logits, every filter: 22 us for the slices (26 MB), 42 for the rows; one row of floats 6 and 27,
// or 77 where a top-p border lies deep in a flat row.  All of it in a row's workgroup, histogram and sums over the whole row: 88 and 104 us; a search for
// the borders bit by bit: 2921 and 3073.
#include <climits>

#include "operators.h"

namespace he_op {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;  // (sixteen wavefronts have too few registers each, and wait longer for one another)
constexpr int kUnit = 42 * 1024;                // log2 of the largest weight, in 1024ths: weights are in units of 2^-42
constexpr int kStep = 4, kBins = ((kUnit + 1024) >> kStep) + 1;  // steps of 2^kStep / 1024 in log2, down to a weight of half a unit
constexpr int kList = 2048;                     // tokens of a step that are compared one with another
constexpr int kHead = 8192;                     // tokens of a row's head
constexpr int kSpans = kThreads;                // spans of ids
constexpr int kSlice = 4096, kSliceThreads = 256, kSliceHead = 2048;
constexpr int kAllHead = 512;                   // a vocabulary of no more is all head
static_assert((1 << 20) / kSlice <= kThreads, "a thread to a slice of the longest row");

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
    float head_logit[kHead];
    int head_id[kHead];
    int slice_n[kThreads];
    unsigned long long wave_u[kWaves], wave_u2[kWaves];
    double wave_d[kWaves];
    float wave_f[kWaves];
    int wave_i[kWaves];
    double before;
    int bin, list_n, head_n, id;
    unsigned long long before_count, before_mass, last, kept_mass;
};

// (z - max) log2(e) / T + 42 in 1024ths: what of it is whole and what is left of it, up to half a 1024th.  Zero: less than half a unit
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

// A row in pieces of 16 bytes from its first value on (they need not lie on 16 bytes).  The last piece ends with the row: it begins with values that the
// one before it has already, which count as -infinity.  (Code is short here and in what follows, loops rather than copies of them: a workgroup goes
// through it a few times, and 150 KB of it, out of memory, took longer than the work.)
template <class E>
struct Row {
    typedef typename E::T T;
    static constexpr int N = 16 / sizeof(T), M = 8, PIECES = M / N;  // values of a piece, handed out at a time
    const T* z;
    int vocab, per_wave, pieces;
    bool infinite;  // the largest logit is +infinity: such tokens weigh the same, the others nothing
    __device__ __forceinline__ Row(const T* p, int v) : z(p), vocab(v), infinite(false) {
        pieces = (vocab + N - 1) / N;
        per_wave = ((pieces + kWaves - 1) / kWaves + 63) & ~63;
    }
    __device__ __forceinline__ int first(int piece) const { return min(piece * N, vocab - N); }  // id of its first value (vocab >= N)
    __device__ __forceinline__ u32x4 raw(int piece) const {
        u32x4 w;
        __builtin_memcpy(&w, z + first(piece), 16);
        return w;
    }
    // have: the piece is there
    __device__ __forceinline__ void values(const u32x4& w, int piece, bool have, float* x) const {
        if constexpr (N == 4) {
            x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
        } else {
            x[0] = E::lo(w.x); x[1] = E::hi(w.x); x[2] = E::lo(w.y); x[3] = E::hi(w.y);
            x[4] = E::lo(w.z); x[5] = E::hi(w.z); x[6] = E::lo(w.w); x[7] = E::hi(w.w);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = fmaxf(x[e], -INFINITY);  // a NaN is never drawn
        if (!have || piece == pieces - 1) {
            const int from = have ? piece * N - first(piece) : N;
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e < from) x[e] = -INFINITY;
        }
        if (infinite) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = x[e] == INFINITY ? 0.f : -INFINITY;
        }
    }
    // f(ids, logits) for every eight of the row's values, -infinity where there is none: contiguous spans of ids to a wavefront
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, end = min(pieces, (wave + 1) * per_wave);
        u32x4 next[PIECES];
#pragma unroll
        for (int x = 0; x < PIECES; ++x) next[x] = raw(min(wave * per_wave + lane + x * 64, pieces - 1));
#pragma unroll 1
        for (int p0 = wave * per_wave; p0 < end; p0 += PIECES * 64) {
            float v[M];
            int id[M];
#pragma unroll
            for (int x = 0; x < PIECES; ++x) {
                const int piece = p0 + lane + x * 64;
                values(next[x], piece, piece < end, v + x * N);
                next[x] = raw(min(piece + PIECES * 64, pieces - 1));
#pragma unroll
                for (int e = 0; e < N; ++e) id[x * N + e] = first(piece) + e;
            }
            f(id, v);
        }
    }
};
// The head of a row, in no order
struct Head {
    static constexpr int M = 4;
    const Shared* sh;
    int n;
    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
        for (int i = threadIdx.x; i < n; i += M * kThreads) {
            float v[M];
            int id[M];
#pragma unroll
            for (int x = 0; x < M; ++x) {
                const int at = i + x * kThreads;
                v[x] = at < n ? sh->head_logit[at] : -INFINITY;
                id[x] = at < n ? sh->head_id[at] : 0;
            }
            f(id, v);
        }
    }
};
// Weights of M logits, all of them worked out side by side (a branch to each would wait for the table M times)
template <int M>
__device__ __forceinline__ void weights(const float* x, double top, double rate, const double* pow2, Log (&l)[M], unsigned long long (&w)[M]) {
#pragma unroll
    for (int e = 0; e < M; ++e) l[e] = log_weight(x[e], top, rate);
#pragma unroll
    for (int e = 0; e < M; ++e) w[e] = weight(l[e], pow2);
}

// The place of the last token kept, of a filter whose border lies in step `bin`: before it `before` tokens' count (or weight) comes from larger
// steps, and the border is the first token at which it reaches `goal`.  Also leaves the weight up to and including that token in sh.kept_mass.
template <class Source>
__device__ __forceinline__ uint64_t border(Shared& sh, const Source& src, double top, double rate, int bin, bool by_count,
                                           unsigned long long before_count, unsigned long long before_mass, double goal) {
    __syncthreads();
    if (threadIdx.x == 0) sh.list_n = 0;
    __syncthreads();
    // the step's logits lie between these: its ends, and a tenth of a 1024th and a rounding more
    float low = (float)(top - ((double)((bin + 1) << kStep) + 0.6) / rate), high = (float)(top - ((double)(bin << kStep) - 0.6) / rate);
    low -= 1e-6f * fabsf(low);
    high += 1e-6f * fabsf(high);
    auto of_bin = [&](auto f) {
        src.each([&](const int (&id)[Source::M], const float (&x)[Source::M]) {
            bool any = false;
#pragma unroll
            for (int e = 0; e < Source::M; ++e) any |= x[e] >= low && x[e] <= high;
            if (!any) return;
#pragma unroll
            for (int e = 0; e < Source::M; ++e) {
                const Log l = log_weight(x[e], top, rate);
                if (!l.zero && (kUnit - l.whole) >> kStep == bin) f(id[e], x[e], l);
            }
        });
    };
    unsigned long long ones = ~0ull, any = 0;
    of_bin([&](int i, float x, const Log& l) {
        const unsigned long long p = place(x, i);
        const int at = atomicAdd(&sh.list_n, 1);
        if (at < kList) {
            sh.list_place[at] = p;
            sh.list_weight[at] = weight(l, sh.pow2);
        }
        ones &= p;
        any |= p;
    });
    __syncthreads();
    const int n = sh.list_n;
    if (n <= kList) {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const unsigned long long mine = sh.list_place[i], w = sh.list_weight[i];
            unsigned long long count = before_count, mass = before_mass;
#pragma unroll 4
            for (int j = 0; j < n; ++j) {
                const bool ahead = sh.list_place[j] > mine;
                count += ahead ? 1 : 0;
                mass += ahead ? sh.list_weight[j] : 0ull;
            }
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
    ones = block_all(ones, sh.wave_u, [](unsigned long long a, unsigned long long b) { return a & b; });
    any = block_all(any, sh.wave_u, [](unsigned long long a, unsigned long long b) { return a | b; });
    const int bits = 64 - __clzll((long long)(ones ^ any));  // (they differ: ids do)
    unsigned long long last = bits == 64 ? 0ull : ones >> bits << bits;
#pragma unroll 1
    for (int b = bits; b >= 0; --b) {  // (first of all the step as a whole, which is known to reach the goal)
        const unsigned long long c = b == bits ? last : last | 1ull << b;
        unsigned long long count = 0, mass = 0;
        of_bin([&](int i, float x, const Log& l) {
            if (place(x, i) >= c) {
                ++count;
                mass += weight(l, sh.pow2);
            }
        });
        count = before_count + block_all(count, sh.wave_u, addu);
        mass = before_mass + block_all(mass, sh.wave_u, addu);
        if (by_count ? (double)count >= goal : (double)mass >= goal) {
            last = c;
            if (threadIdx.x == 0) sh.kept_mass = mass;
        }
    }
    __syncthreads();
    return last;
}

struct Ask {  // a row's filters, and what is known of it
    double top, rate;
    float topf, p, least;
    int k;
    bool top_k, top_p;
};
struct Limit { float z; int id; bool all; };  // kept: logits above z, and equal to it up to id; all: nothing below the source is

// What the filters keep of a source's tokens and of those below them that it does not hold, whose weights are `below` in all (`complete`: there are
// none of any weight).
template <class Source>
__device__ __forceinline__ Limit limit_of(Shared& sh, const Source& src, const Ask& ask, unsigned long long below, bool complete, float cut) {
    constexpr int M = Source::M;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Limit lim{-INFINITY, INT_MAX, complete};
    bool undecided = false;
    if (ask.top_k || ask.top_p) {
        for (int i = threadIdx.x; i < kBins; i += kThreads) { sh.mass[i] = 0; sh.count[i] = 0; }
        __syncthreads();
        src.each([&](const int (&)[M], const float (&x)[M]) {
            Log l[M];
            unsigned long long w[M];
            weights<M>(x, ask.top, ask.rate, sh.pow2, l, w);
#pragma unroll
            for (int e = 0; e < M; ++e) {
                const int bin = l[e].zero ? kBins - 1 : (kUnit - l[e].whole) >> kStep;
                atomicAdd(&sh.mass[bin], w[e]);
                if (ask.top_k) atomicAdd(&sh.count[bin], l[e].zero ? 0u : 1u);
            }
        });
        __syncthreads();
        // running sums over the steps, six to a thread, in their places
        constexpr int PER = (kBins + kThreads - 1) / kThreads;
        {
            unsigned int cs = 0;
            unsigned long long ms = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = threadIdx.x * PER + i;
                if (at < kBins) { cs += sh.count[at]; ms += sh.mass[at]; }
            }
            const unsigned long long cu = wave_upto(cs), mu = wave_upto(ms);
            if (lane == 63) { sh.wave_u[wave] = cu; sh.wave_u2[wave] = mu; }
            __syncthreads();
            unsigned long long c = cu - cs, m = mu - ms;  // before this thread's steps
            for (int w = 0; w < wave; ++w) { c += sh.wave_u[w]; m += sh.wave_u2[w]; }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = threadIdx.x * PER + i;
                if (at < kBins) {
                    sh.count[at] = (unsigned int)(c += sh.count[at]);
                    sh.mass[at] = m += sh.mass[at];
                }
            }
            __syncthreads();
        }
        const unsigned long long c_all = sh.count[kBins - 1], m_all = sh.mass[kBins - 1];
        uint64_t last = 0;
        unsigned long long of_first = m_all + below;  // weight of the first k
        const bool k_here = ask.top_k && c_all >= (unsigned long long)ask.k;
        undecided = ask.top_p && ask.top_k && !k_here && !complete;  // (a share of the first k's weight, of which some lie below)
        for (int by_count = 1; by_count >= 0; --by_count) {
            const double goal = by_count ? (double)ask.k : (double)ask.p * (double)of_first;
            if (by_count ? !k_here : !ask.top_p || undecided || goal > (double)m_all) continue;
            for (int i = threadIdx.x; i < kBins; i += kThreads) {
                const unsigned long long cb = i ? sh.count[i - 1] : 0, mb = i ? sh.mass[i - 1] : 0;
                if ((double)(by_count ? cb : mb) < goal && (double)(by_count ? sh.count[i] : sh.mass[i]) >= goal) {
                    sh.bin = i;
                    sh.before_count = cb;
                    sh.before_mass = mb;
                }
            }
            __syncthreads();
            const uint64_t at = border(sh, src, ask.top, ask.rate, sh.bin, by_count, sh.before_count, sh.before_mass, goal);
            last = at > last ? at : last;
            lim.all = true;
            of_first = sh.kept_mass;
            __syncthreads();
        }
        if (last) {
            lim.z = place_logit(last);
            lim.id = (int)~(uint32_t)last;
        }
    }
    if (ask.least > 0.f) {
        // w >= min_p as a bound on the logit, up to the next float
        const double bound = ask.top + log2((double)ask.least) * 1024.0 / ask.rate;
        float b = (float)bound;
        if ((double)b < bound) b = nextafterf(b, INFINITY);
        if (b > lim.z) { lim.z = fminf(b, ask.topf); lim.id = INT_MAX; }
        if (b >= cut) lim.all = true;
    }
    lim.all &= !undecided;
    return lim;
}

// ---- the slices
//
// What a slice's workgroup leaves.  soft, rest, mass: sums of exp(z - largest) and of exp((z - largest) / T) -- soft and rest over the tokens below
// `cut`, mass, of a row without filters, over all of them.
struct Slice {
    float largest, cut;
    int n, whole;  // tokens of the head; whole: it did not fit, and the row is gone over as a whole
    double soft, rest, mass;
};
struct Workspace {
    Slice* slices;  // [rows][n_slices]
    float* logit;   // [rows][n_slices][kSliceHead]
    int* id;
};
__host__ __device__ inline int slices_of(int vocab) { return (vocab + kSlice - 1) / kSlice; }
__host__ __device__ inline Workspace workspace_of(void* p, int rows, int vocab) {
    const size_t n = (size_t)rows * slices_of(vocab);
    Workspace w;
    w.slices = reinterpret_cast<Slice*>(p);
    w.logit = reinterpret_cast<float*>(w.slices + n);
    w.id = reinterpret_cast<int*>(w.logit + n * kSliceHead);
    return w;
}

struct RowFilters {
    float temperature, p, least;
    int k;
    bool first_only, top_k, top_p, any;
};
__device__ __forceinline__ RowFilters filters_of(const Filters& f, int r, int vocab) {
    RowFilters a;
    a.temperature = f.temperature ? f.temperature[r] : 1.f;
    a.k = f.top_k ? f.top_k[r] : 0;
    a.p = f.top_p ? f.top_p[r] : 1.f;
    a.least = f.min_p ? f.min_p[r] : 0.f;
    a.first_only = a.k == 1 || !(a.temperature > 0.f) || a.p <= 0.f || a.least > 1.f;
    a.top_k = !a.first_only && a.k > 1 && a.k < vocab;
    a.top_p = !a.first_only && a.p < 1.f;
    a.any = a.first_only || a.top_k || a.top_p || a.least > 0.f || vocab <= kAllHead;  // (a row that is all head)
    return a;
}

template <class E>
__global__ __launch_bounds__(kSliceThreads) void slice_kernel(Rows logits, int vocab, Filters f, Workspace ws) {
    typedef typename E::T T;
    constexpr int N = Row<E>::N, P = kSlice / kSliceThreads / N, W = kSliceThreads / 64;  // pieces to a thread
    __shared__ float sh_max[W], sh_cut[W];
    __shared__ int sh_n[W];
    __shared__ double sh_sum[3][W];
    const int r = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const size_t at = (size_t)r * gridDim.x + blockIdx.x;
    const Row<E> row((const T*)logits.data + (int64_t)r * logits.stride, vocab);
    const int piece0 = blockIdx.x * (kSlice / N) + threadIdx.x;
    const RowFilters ask = filters_of(f, r, vocab);
    float x[P * N], best = -INFINITY;
    if (vocab >= N) {
        u32x4 w[P];
#pragma unroll
        for (int i = 0; i < P; ++i) w[i] = row.raw(min(piece0 + i * kSliceThreads, row.pieces - 1));
#pragma unroll
        for (int i = 0; i < P; ++i) row.values(w[i], piece0 + i * kSliceThreads, piece0 + i * kSliceThreads < row.pieces, x + i * N);
    } else {  // (a vocabulary of less than a piece: a token to each of the first threads)
#pragma unroll
        for (int i = 0; i < P * N; ++i) x[i] = -INFINITY;
        if ((int)threadIdx.x < vocab) x[0] = fmaxf(E::up(row.z[threadIdx.x]), -INFINITY);
    }
#pragma unroll
    for (int i = 0; i < P * N; ++i) best = fmaxf(best, x[i]);
    // Each of 128 groups of the slice's tokens has one at `cut` or above it: some 128 (ln 128 + 0.6) = 700, if they lie in no particular order, and hardly
    // ever three times as many.  (Fewer groups to each of many slices, so that a row's heads together fit into LDS.)  Groups of nothing but
    // -infinity do not count.
    float of_group = lane_max<2>(best);
    if (gridDim.x > 16) of_group = fmaxf(of_group, lane_xor2(of_group));
    if (gridDim.x > 32) of_group = fmaxf(of_group, lane_mirror8(of_group));
    if (gridDim.x > 64) of_group = fmaxf(of_group, lane_mirror16(of_group));
    const float other = lane_max<64>(of_group > -INFINITY ? -of_group : -INFINITY);
    best = lane_max<64>(best);
    if (lane == 0) { sh_max[wave] = best; sh_cut[wave] = other; }
    __syncthreads();
    float largest = sh_max[0], cut = sh_cut[0];
#pragma unroll
    for (int i = 1; i < W; ++i) { largest = fmaxf(largest, sh_max[i]); cut = fmaxf(cut, sh_cut[i]); }
    cut = -cut;  // (+infinity where there is nothing)
    if (vocab <= kAllHead) cut = -INFINITY;
    if (largest == INFINITY) cut = INFINITY;
    int mine = 0;
    uint32_t in_head = 0;
#pragma unroll
    for (int i = 0; i < P * N; ++i) in_head |= (uint32_t)(x[i] >= cut && x[i] > -INFINITY) << i;
    mine = __popc(in_head);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 63) sh_n[wave] = upto;
    __syncthreads();
    int n = 0, to = upto - mine;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (i < wave) to += sh_n[i];
        n += sh_n[i];
    }
    const bool whole = n > kSliceHead;
    if (!whole) {
        float* logit = ws.logit + at * kSliceHead;
        int* id = ws.id + at * kSliceHead;
#pragma unroll
        for (int i = 0; i < P * N; ++i)
            if (in_head >> i & 1) {
                logit[to] = x[i];
                id[to] = vocab >= N ? row.first(piece0 + i / N * kSliceThreads) + i % N : (int)threadIdx.x;
                ++to;
            }
    }
    // Sums of the others in float but for the additions: 2^-21 of a term at most, in no one direction (log2 e, and log2 e / T, in two parts); the head's are
    // left to whoever has all of the row.  (-infinity, and differences from an infinite largest, are nothing.)
    double soft = 0.0, rest = 0.0, mass = 0.0;
    if (largest > -INFINITY && largest < INFINITY) {
        const double rate = 1.4426950408889634 / (double)ask.temperature;
        if (!whole) {
            const float hi = (float)rate, lo = (float)(rate - (double)hi);
            float s = 0.f, t = 0.f;
#pragma unroll
            for (int i = 0; i < P * N; ++i) {
                const float d = fmaxf(x[i] - largest, -3e38f);
                const bool in = in_head >> i & 1;
                const float a = __builtin_amdgcn_exp2f(fmaf(d, 1.44269502f, d * 1.92596299e-8f));
                s += in ? 0.f : a;
                if (ask.top_p) t += in ? 0.f : __builtin_amdgcn_exp2f(fmaf(d, hi, d * lo));
            }
            soft = (double)s;
            rest = (double)t;
        }
        if (!ask.any)
#pragma unroll
            for (int i = 0; i < P * N; ++i) {
                const double e = ((double)x[i] - (double)largest) * rate;
                mass += e >= -43.0 ? exp2(e) : 0.0;  // (no NaN of -infinity times nothing, and none that weighs nothing against the row's largest)
            }
    } else if (largest == INFINITY) {  // so many of one weight, and nothing else
        mass = (double)mine;
    }
    const auto addd = [](double a, double b) { return a + b; };
    soft = wave_all(soft, addd);
    rest = wave_all(rest, addd);
    if (!ask.any) mass = wave_all(mass, addd);
    if (lane == 0) { sh_sum[0][wave] = soft; sh_sum[1][wave] = rest; sh_sum[2][wave] = mass; }
    __syncthreads();
    if (threadIdx.x == 0) {
        Slice s{largest, cut, whole ? 0 : n, whole, 0.0, 0.0, 0.0};
#pragma unroll
        for (int i = 0; i < W; ++i) { s.soft += sh_sum[0][i]; s.rest += sh_sum[1][i]; s.mass += sh_sum[2][i]; }
        ws.slices[at] = s;
    }
}

// ---- the rows
template <class E>
__global__ __launch_bounds__(kThreads) void sample_kernel(Rows logits, int vocab, Filters f, Workspace ws, const float* __restrict__ uniform,
                                                          int32_t* __restrict__ ids, float* __restrict__ logprobs) {
    typedef typename E::T T;
    __shared__ Shared sh;
    const int r = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n_slices = slices_of(vocab);
    Row<E> row((const T*)logits.data + (int64_t)r * logits.stride, vocab);
    const auto addu = [](unsigned long long a, unsigned long long b) { return a + b; };
    const auto addd = [](double a, double b) { return a + b; };
    const auto orr = [](int a, int b) { return a | b; };

    Slice mine{-INFINITY, -INFINITY, 0, 0, 0.0, 0.0, 0.0};
    if ((int)threadIdx.x < n_slices) mine = ws.slices[(size_t)r * n_slices + threadIdx.x];
    const RowFilters rf = filters_of(f, r, vocab);
    const float u = uniform[r];
    sh.slice_n[threadIdx.x] = mine.n;
    if (threadIdx.x == 0) { sh.id = INT_MAX; sh.head_n = 0; }
    for (int i = threadIdx.x; i < 1024; i += kThreads) sh.pow2[i] = exp2((double)i / 1024.0);
    const bool some = mine.largest > -INFINITY;
    const float best = block_all(mine.largest, sh.wave_f, [](float a, float b) { return fmaxf(a, b); });
    float cut = block_all(some ? mine.cut : -INFINITY, sh.wave_f, [](float a, float b) { return fmaxf(a, b); });
    const bool whole = block_all((int)mine.whole, sh.wave_i, orr) != 0;
    if (best == -INFINITY) {
        if (threadIdx.x == 0) {
            ids[r] = -1;
            logprobs[r] = -INFINITY;
        }
        return;
    }
    row.infinite = best == INFINITY;
    if (row.infinite) cut = 0.f;
    Ask ask;
    ask.topf = row.infinite ? 0.f : best;
    const double top = ask.top = ask.topf;
    ask.k = rf.k;
    ask.p = rf.p;
    ask.least = rf.least;
    ask.top_k = rf.top_k;
    ask.top_p = rf.top_p;
    constexpr double kPlain = 1024.0 * 1.4426950408889634;
    const double rate = ask.rate = rf.first_only ? kPlain : kPlain / (double)rf.temperature;

    // the sums of what the slices' heads do not hold, and the heads: those from `cut` up into LDS, the others into the sums
    double lse = some && !row.infinite ? mine.soft * exp2(((double)mine.largest - top) * (kPlain / 1024.0)) : 0.0;
    double rest = some && !row.infinite && ask.top_p ? mine.rest * exp2(((double)mine.largest - top) * (rate / 1024.0)) : 0.0;
    int first = INT_MAX;
    // (a slice to a wavefront, sixteen tokens to a lane on their way together; those below the cut count in float, like the slices' sums)
    const float rate_hi = (float)(rate / 1024.0), rate_lo = (float)(rate / 1024.0 - (double)rate_hi);
#pragma unroll 1
    for (int s = wave; s < n_slices; s += kWaves) {
        constexpr int B = 16;
        const int n = sh.slice_n[s];
        const size_t at = ((size_t)r * n_slices + s) * kSliceHead + lane;
        float soft_part = 0.f, rest_part = 0.f;
#pragma unroll 1
        for (int i0 = 0; i0 < n; i0 += B * 64) {
            float x[B];
            int id[B];
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const bool have = i0 + i * 64 + lane < n;
                x[i] = have ? ws.logit[at + i0 + i * 64] : -INFINITY;
                id[i] = have ? ws.id[at + i0 + i * 64] : 0;
            }
#pragma unroll
            for (int i = 0; i < B; ++i) {
                if (row.infinite) x[i] = x[i] == INFINITY ? 0.f : -INFINITY;
                const bool in = x[i] >= cut && x[i] > -INFINITY;
                const float d = fmaxf(x[i] - ask.topf, -3e38f);
                const float a = __builtin_amdgcn_exp2f(fmaf(d, 1.44269502f, d * 1.92596299e-8f));
                soft_part += in ? 0.f : a;
                if (ask.top_p) {
                    const float t = __builtin_amdgcn_exp2f(fmaf(d, rate_hi, d * rate_lo));
                    rest_part += in ? 0.f : t;
                }
                const uint64_t who = __ballot(in);
                int base = 0;
                if (lane == 0) base = atomicAdd(&sh.head_n, __popcll(who));
                base = __builtin_amdgcn_readfirstlane(base) + __popcll(who & ((1ull << lane) - 1));
                if (in && base < kHead) { sh.head_logit[base] = x[i]; sh.head_id[base] = id[i]; }
                if (in && x[i] == ask.topf) first = min(first, id[i]);
            }
        }
        lse += (double)soft_part;
        rest += (double)rest_part;
    }
    __syncthreads();
    Head head{&sh, min(sh.head_n, kHead)};
    const bool whole_head = !whole && sh.head_n <= kHead;
    // the head's own part of the soft-max's sum: a few large terms can be all of it
    if (whole_head) {
        head.each([&](const int (&)[4], const float (&x)[4]) {
            Log l[4];
            unsigned long long w[4];
            weights<4>(x, top, kPlain, sh.pow2, l, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) lse += (double)w[i] * 0x1p-42;
        });
    } else {  // (it does not fit: all of the row)
        lse = 0.0;
        row.each([&](const int (&)[8], const float (&x)[8]) {
            Log l[8];
            unsigned long long w[8];
            weights<8>(x, top, kPlain, sh.pow2, l, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) lse += (double)w[i] * 0x1p-42;
        });
    }
    lse = block_all(lse, sh.wave_d, addd);
    rest = block_all(rest, sh.wave_d, addd);
    int id = -1;
    const double want = u > 0.f ? (double)u : 0.0;
    if (rf.first_only && !whole) {
        if (first != INT_MAX) atomicMin(&sh.id, first);
        __syncthreads();
        if (threadIdx.x == 0) id = sh.id;
    } else if (!rf.any) {
        // no filters: the slice in which the number falls, and the place in it
        double m = mine.mass * (some && !row.infinite ? exp2(((double)mine.largest - top) * (rate / 1024.0)) : 1.0), upto = m;
        if (row.infinite && mine.largest < INFINITY) upto = m = 0.0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        __syncthreads();  // (everybody has the sums above)
        if (lane == 63) sh.wave_d[wave] = upto;
        if (threadIdx.x == 0) { sh.bin = -1; sh.list_n = -1; }
        __syncthreads();
        double total = 0.0, base = 0.0;
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) base = total;
            total += sh.wave_d[w];
        }
        upto += base;
        const double goal = want * total;
        // (the last slice of any weight that begins at the number or below it: sums of several, so that every number has one)
        if (m > 0.0 && upto - m <= goal) atomicMax(&sh.bin, (int)threadIdx.x);
        __syncthreads();
        const int s = max(sh.bin, 0);
        if ((int)threadIdx.x == s) sh.before = upto - m;
        __syncthreads();
        constexpr int N = Row<E>::N, P = kSlice / kThreads / N;  // pieces to a thread, one behind the other
        float x[P * N];
        const int piece0 = s * (kSlice / N) + threadIdx.x * P;
#pragma unroll
        for (int i = 0; i < P; ++i) row.values(row.raw(min(piece0 + i, row.pieces - 1)), piece0 + i, piece0 + i < row.pieces, x + i * N);
        auto id_of = [&](int i) { return row.first(piece0 + i / N) + i % N; };
        Log l[P * N];
        unsigned long long w[P * N], sum = 0;
        weights<P * N>(x, top, rate, sh.pow2, l, w);
        int last = -1;
#pragma unroll
        for (int i = 0; i < P * N; ++i) {
            sum += w[i];
            if (w[i]) last = id_of(i);
        }
        if (last >= 0) atomicMax(&sh.list_n, last);
        unsigned long long after = wave_upto(sum);
        if (lane == 63) sh.wave_u[wave] = after;
        __syncthreads();
        unsigned long long all = 0;
        for (int v = 0; v < kWaves; ++v) {
            if (v < wave) after += sh.wave_u[v];
            all += sh.wave_u[v];
        }
        const double in_slice = fmax(goal - sh.before, 0.0) * 4398046511104.0;  // 2^42
        if (!(in_slice < (double)all)) {
            if (threadIdx.x == 0) id = sh.list_n;  // a number of 1 or more, or a rounding's worth past the slice: its last token
        } else if ((double)(after - sum) <= in_slice && (double)after > in_slice) {  // (one thread)
            unsigned long long c = after - sum;
#pragma unroll
            for (int i = 0; i < P * N; ++i) {
                c += w[i];
                if (id < 0 && (double)c > in_slice) id = id_of(i);
            }
        }
    } else {
        Limit lim{-INFINITY, INT_MAX, false};
        bool by_head = false;
        if (rf.first_only) {
            lim.z = ask.topf;  // (more than fit of one value or little else: its first, below)
        } else {
            if (whole_head && (rate < 1e30 || vocab <= kAllHead)) {  // (a temperature next to nothing: the rest's weights are no floats)
                const bool complete = row.infinite || vocab <= kAllHead || log_weight(cut, top, rate).zero;
                lim = limit_of(sh, head, ask, (unsigned long long)(rest * 4398046511104.0), complete, cut);
                by_head = lim.all;
            }
            if (!by_head) {
                __syncthreads();
                lim = limit_of(sh, row, ask, 0, true, -INFINITY);
            }
        }
        auto kept = [&](float x, int i) { return x > lim.z || (x == lim.z && i <= lim.id); };
        if (by_head) {
            // the kept weights by spans of ids; the span in which the number falls; and its tokens, each adding up those of lower ids
            int shift = 0;
            while ((vocab - 1) >> shift >= kSpans) ++shift;
            __syncthreads();
            sh.mass[threadIdx.x] = 0;
            if (threadIdx.x == 0) { sh.id = -1; sh.list_n = 0; }
            __syncthreads();
            int final = -1;
            head.each([&](const int (&i)[4], const float (&x)[4]) {
                if (fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) < lim.z) return;
                Log l[4];
                unsigned long long w[4];
                weights<4>(x, top, rate, sh.pow2, l, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = w[e] && kept(x[e], i[e]);
                    atomicAdd(&sh.mass[i[e] >> shift], in ? w[e] : 0ull);
                    final = max(final, in ? i[e] : -1);
                }
            });
            if (final >= 0) atomicMax(&sh.id, final);
            __syncthreads();
            const unsigned long long m = sh.mass[threadIdx.x];
            unsigned long long upto = wave_upto(m), total = 0;
            if (lane == 63) sh.wave_u[wave] = upto;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) upto += sh.wave_u[w];
                total += sh.wave_u[w];
            }
            const double goal = want * (double)total;
            if (!(goal < (double)total)) {  // a number of 1 or more: the last token kept
                if (threadIdx.x == 0) id = sh.id;
            } else {
                if ((double)(upto - m) <= goal && (double)upto > goal) { sh.bin = threadIdx.x; sh.before_mass = upto - m; }  // (one thread)
                __syncthreads();
                const int span = sh.bin;
                head.each([&](const int (&i)[4], const float (&x)[4]) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (x[e] > -INFINITY && i[e] >> shift == span && kept(x[e], i[e])) {
                            const int at = atomicAdd(&sh.list_n, 1);  // (a span has 2048 ids at most)
                            sh.list_place[at] = (unsigned long long)i[e];
                            sh.list_weight[at] = weight(log_weight(x[e], top, rate), sh.pow2);
                        }
                });
                __syncthreads();
                const int n = sh.list_n;
                for (int i = threadIdx.x; i < n; i += kThreads) {
                    const unsigned long long me = sh.list_place[i];
                    unsigned long long sum = sh.before_mass;
                    for (int j = 0; j < n; ++j) sum += sh.list_place[j] < me ? sh.list_weight[j] : 0ull;
                    if ((double)sum <= goal && (double)(sum + sh.list_weight[i]) > goal) id = (int)me;
                }
            }
        } else {
            constexpr int M = Row<E>::M, N = Row<E>::N;
            unsigned long long sum = 0;
            int final = -1, lowest = INT_MAX;
            row.each([&](const int (&i)[M], const float (&x)[M]) {
                bool any = false;
#pragma unroll
                for (int e = 0; e < M; ++e) any |= x[e] >= lim.z;
                if (!any) return;
                Log l[M];
                unsigned long long w[M];
                weights<M>(x, top, rate, sh.pow2, l, w);
#pragma unroll
                for (int e = 0; e < M; ++e) {
                    const bool in = w[e] && kept(x[e], i[e]);
                    sum += in ? w[e] : 0ull;
                    final = max(final, in ? i[e] : -1);
                    lowest = min(lowest, in ? i[e] : INT_MAX);
                }
            });
            if (rf.first_only) {  // (nothing is above the limit)
                if (threadIdx.x == 0) sh.id = INT_MAX;
                __syncthreads();
                if (lowest != INT_MAX) atomicMin(&sh.id, lowest);
                __syncthreads();
                if (threadIdx.x == 0) id = sh.id;
            } else {
                const unsigned long long of_wave = wave_all(sum, addu);
                const int last_id = wave_all(final, [](int a, int b) { return max(a, b); });
                __syncthreads();
                if (lane == 0) { sh.wave_u[wave] = of_wave; sh.wave_i[wave] = last_id; }
                __syncthreads();
                unsigned long long before = 0, total = 0;
                for (int w = 0; w < kWaves; ++w) {
                    if (w < wave) before += sh.wave_u[w];
                    total += sh.wave_u[w];
                }
                const double goal = want * (double)total;
                if (!(goal < (double)total)) {
                    if (threadIdx.x == 0)
                        for (int w = 0; w < kWaves; ++w) id = max(id, sh.wave_i[w]);
                } else if ((double)before <= goal && (double)(before + of_wave) > goal) {  // (one wavefront)
                    const int end = min(row.pieces, (wave + 1) * row.per_wave);
                    for (int p0 = wave * row.per_wave; p0 < end; p0 += 64) {
                        float x[N];
                        Log l[N];
                        unsigned long long w[N], of_lane = 0;
                        const int piece = p0 + lane, i0 = row.first(piece);
                        row.values(row.raw(min(piece, row.pieces - 1)), piece, piece < end, x);
                        weights<N>(x, top, rate, sh.pow2, l, w);
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            w[e] = kept(x[e], i0 + e) ? w[e] : 0ull;
                            of_lane += w[e];
                        }
                        const unsigned long long upto = before + wave_upto(of_lane);
                        if ((double)(upto - of_lane) <= goal && (double)upto > goal) {  // (one lane)
                            unsigned long long c = upto - of_lane;
#pragma unroll
                            for (int e = 0; e < N; ++e) {
                                c += w[e];
                                if (id < 0 && (double)c > goal) id = i0 + e;
                            }
                        }
                        if (__any(id >= 0)) break;
                        before = __shfl(upto, 63);
                    }
                }
            }
        }
    }
    if (id >= 0) {
        const float logit = fmaxf(E::up(row.z[id]), -INFINITY);
        ids[r] = id;
        logprobs[r] = (float)((row.infinite ? 0.0 : (double)logit - top) - log(lse));
    }
}

}  // namespace

size_t sample_workspace(int rows, int vocab) { return (size_t)rows * slices_of(vocab) * (sizeof(Slice) + kSliceHead * 8); }

void sample(hipStream_t s, he_dtype dt, Rows logits, int rows, int vocab, const Filters& f, const float* uniform, int32_t* ids, float* logprobs,
            void* workspace) {
    by_type(dt, [&](auto e) {
        typedef decltype(e) E;
        const Workspace ws = workspace_of(workspace, rows, vocab);
        slice_kernel<E><<<dim3(slices_of(vocab), rows), kSliceThreads, 0, s>>>(logits, vocab, f, ws);
        sample_kernel<E><<<rows, kThreads, 0, s>>>(logits, vocab, f, ws, uniform, ids, logprobs);
    });
}

}  // namespace he_op
