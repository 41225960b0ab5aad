// Attention of GQ queries that share their keys, by a workgroup of four wavefronts on the vector units, in one pass over the keys.
//
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q . k_j,  m = max_j s_j
//
// DP/8 adjacent lanes own a key (eight dimensions each, DP the head dimension rounded up to a power of two: lanes past the
// head dimension hold zeros), and keep the running maximum, sum and weighted values of the keys they have seen, in float; K and V of the
// next round are on their way meanwhile.  The lanes of a wavefront are merged by data-parallel moves, the wavefronts through LDS.
#pragma once
#include "operators.h"

namespace he_op {

template <int DP, int GQ>
struct AttendShared {
    float2 ml[4][GQ];
    float o[4][GQ][DP];
};

// rows(j, k, v): whether key j counts, and where its K and V rows begin.  qs: the queries' eight dimensions of this lane, times the scale.
// emit(g, e, m, l, o): called once for every query g and dimension e < DP, by the thread that holds it: maximum, sum, weighted value.
template <class E, int DP, int GQ, class RowsOf, class Emit>
__device__ __forceinline__ void attend(AttendShared<DP, GQ>& sh, int begin, int end, int d, const float (&qs)[GQ][8], RowsOf rows, Emit emit) {
    typedef typename E::T T;
    constexpr int LPK = DP / 8, KPW = 64 / LPK, KR = 4 * KPW, U = sizeof(T) == 4 || GQ > 2 ? 2 : 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, sub = lane % LPK, jw = wave * KPW + lane / LPK;
    const bool in_row = sub * 8 < d;
    Raw8<E> k[U], v[U];
    bool ok[U];
    auto request = [&](int base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = base + u * KR + jw;
            const T *kp, *vp;
            ok[u] = j < end && rows(j, kp, vp);
            k[u] = v[u] = zero8<E>();
            if (ok[u] && in_row) {
                k[u] = load8<E>(kp + sub * 8);
                v[u] = load8<E>(vp + sub * 8);
            }
        }
    };
    float m[GQ], l[GQ], acc[GQ][8];
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
        m[g] = -INFINITY;
        l[g] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[g][e] = 0.f;
    }
    request(begin);
    for (int base = begin; base < end; base += U * KR) {
        float kf[U][8], vf[U][8];
        bool now[U];
#pragma unroll
        for (int u = 0; u < U; ++u) { unpack8<E>(k[u], kf[u]); unpack8<E>(v[u], vf[u]); now[u] = ok[u]; }
        if (base + U * KR < end) request(base + U * KR);
#pragma unroll
        for (int g = 0; g < GQ; ++g) {
            float s[U], top = m[g];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x = fmaf(qs[g][e], kf[u][e], x);
                x = lane_sum<LPK>(x);
                s[u] = now[u] ? x : -INFINITY;
                // (a NaN score is nobody's maximum, and makes its row NaN through the sum)
                top = fmaxf(top, s[u]);
            }
            const float ref = top > -INFINITY ? top : 0.f, keep = expf(m[g] - ref);
            m[g] = top;
            l[g] *= keep;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[g][e] *= keep;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float p = now[u] ? expf(s[u] - ref) : 0.f;
                l[g] += p;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[g][e] = fmaf(p, vf[u][e], acc[g][e]);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
        float top = m[g];
        if (LPK <= 8) top = fmaxf(top, lane_xor8(top));
        if (LPK <= 16) top = lane_max16_apart(top);
        top = lane_max32_apart(top);
        const float own = m[g] > -INFINITY ? expf(m[g] - top) : l[g];  // (l is 0 there, or NaN)
        const float sum = lane_sum_apart<LPK>(l[g] * own);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[g][e] = lane_sum_apart<LPK>(acc[g][e] * own);
        if (lane == 0) sh.ml[wave][g] = make_float2(top, sum);
        if (lane < LPK) {
            float4* dst = reinterpret_cast<float4*>(&sh.o[wave][g][sub * 8]);
            dst[0] = make_float4(acc[g][0], acc[g][1], acc[g][2], acc[g][3]);
            dst[1] = make_float4(acc[g][4], acc[g][5], acc[g][6], acc[g][7]);
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < GQ * DP; x += 256) {
        const int g = x / DP, e = x % DP;
        float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sh.ml[w][g].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 a = sh.ml[w][g];
            const float f = a.x > -INFINITY ? expf(a.x - top) : a.y;
            sum += a.y * f;
            o += sh.o[w][g][e] * f;
        }
        emit(g, e, top, sum, o);
    }
}

// The lane's eight dimensions of a query, times the scale
template <class E, int DP>
__device__ __forceinline__ void query8(const typename E::T* p, int d, float scale, float (&q)[8]) {
    const int sub = (threadIdx.x & 63) % (DP / 8);
    float f[8];
    unpack8<E>(sub * 8 < d ? load8<E>(p + sub * 8) : zero8<E>(), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = f[e] * scale;
}

// Result of a row that saw no key: zeros
__device__ __forceinline__ float attended(float l, float o) { return l == 0.f ? 0.f : o / l; }

}  // namespace he_op
