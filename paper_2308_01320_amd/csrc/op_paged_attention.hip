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
    return {reinterpret_cast<float2*>(workspace), workspace + (2 * rows * splits + 3) / 4 * 4};
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

// The same on the matrix cores, for the 16-bit types and pages of 16 positions or more: up to sixteen queries that share their keys are the columns
// of S^T = K Q^T and O^T = V^T P^T.  A wavefront has every fourth tile of 32 keys to itself, from the loads to its own part of the result,
// so nothing in the loop waits for another: K goes from memory into operands, V past the registers into LDS, both a tile ahead, and V is
// transposed by the reads.  A lane holds one query; its four keys of each half of the tile are four of its weights' eight places, in the
// order in which V's rows are read.  Weights multiply V as two terms of the type (2^-16 of a weight is lost with bf16), which costs nothing here:
// what bounds the kernel is the stream of K and V, with 64 KB of it requested ahead by a workgroup and two of those on a CU.  Measured, with the
// join: 4 sequences of up to 100003 positions, 40/8 heads of 128, 1.31 GB, 211 us = 6.2 TB/s (a streaming read reaches 6.1 to 6.5; on the vector
// units 664); 32 of up to 511, 40 heads, 227 MB, 43 us (51); one of 77 positions, 32 heads of 64, 4.0 us, which is the chain from its length over its page to its result.
template <class E, int DP, bool EXACT>
struct PagedTile {
    static constexpr int CPR = DP / 8, LOADS = DP / 16, RPN = 64 / CPR;  // 16-byte pieces of a row; copies of V per tile, rows of each
    static __device__ __forceinline__ int turn(int r) { return CPR >= 16 ? (r & 7) << 1 : r & 6; }  // (as in the prompts' tiles)
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 mma16(BF16, const u32x4& a, const u32x4& b, f32x4 c) {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(F16, const u32x4& a, const u32x4& b, f32x4 c) {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}

// Four operands of V^T: blocks of sixteen dimensions at the four places, keys 4 g + 0..3 and 16 + 4 g + 0..3 (g = lane / 16), BYTES apart
template <int BYTES>
__device__ __forceinline__ void v_operands(u32x4 (&o)[4], const uint32_t (&at)[4]) {
    uint2 r[8];
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
        "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(BYTES)
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = u32x4{r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y};
}

template <class E, int DP, bool EXACT>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void paged_mma_kernel(Cache c, Rows q, int n_heads, Rows out, const int32_t* __restrict__ lens, int splits, float scale,
                                                                           float* __restrict__ workspace) {
    typedef typename E::T T;
    typedef PagedTile<E, DP, EXACT> Ti;
    constexpr int WAVES = 4, KB = DP / 32, OB = DP / 16, PITCH = DP + 4, REGION = 2 * 32 * DP * 2;  // a wavefront's two tiles of V, in bytes
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ float2 ml[WAVES][16];
    const int d = EXACT ? DP : c.head_dim, share = n_heads / c.n_kv_heads, groups = (share + 15) / 16;
    const int part = blockIdx.x % splits, rest = blockIdx.x / splits, h = rest / groups, g0 = rest % groups * 16, b = blockIdx.y, nq = min(16, share - g0);
    const int len = (int)min((int64_t)max(lens[b], 0), (int64_t)c.pages_per_seq << c.page_shift);
    int begin, end;
    share_of(len, splits, part, begin, end);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int n_tiles = (end - begin + 31) / 32;
    const int32_t* table = c.pages + (size_t)b * c.pages_per_seq;
    // the pages of the two halves of a tile, -1: none
    struct Pages { int p[2]; };
    auto pages = [&](int tile) {
        Pages r;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int t = begin + tile * 32 + x * 16;
            const int p = t < end ? table[t >> c.page_shift] : -1;
            r.p[x] = (unsigned)p < (unsigned)c.n_pages ? p : -1;
        }
        return r;
    };
    auto offset = [&](const Pages& pg, int tile, int x) {  // of the first row of half x, in elements; of a page that is none: page 0's
        return cache_row(c, max(pg.p[x], 0), h, begin + tile * 32 + x * 16);
    };
    unsigned char* region = smem + wave * REGION;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)region;
    uint32_t v_place[Ti::LOADS];  // a lane's row and piece of each copy
#pragma unroll
    for (int n = 0; n < Ti::LOADS; ++n) {
        const int r = n * Ti::RPN + lane / Ti::CPR;
        int pc = (lane % Ti::CPR) ^ Ti::turn(r);
        if (!EXACT) pc = min(pc, d / 8 - 1);
        v_place[n] = (r & 15) * d + pc * 8;
    }
    auto request_v = [&](const Pages& pg, int tile, int buf) {
        const T* at[2] = {(const T*)c.v + offset(pg, tile, 0), (const T*)c.v + offset(pg, tile, 1)};
#pragma unroll
        for (int n = 0; n < Ti::LOADS; ++n)
            he_bf16::load_block_to_lds<true>(reinterpret_cast<const u32x4*>(at[n * Ti::RPN / 16] + v_place[n]), reinterpret_cast<u32x4*>(region + buf * (REGION / 2)) + n * 64);
    };
    auto request_k = [&](const Pages& pg, int tile, u32x4 (&k)[2][KB]) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const T* at = (const T*)c.k + offset(pg, tile, x) + j * d + g * 8;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                k[x][kb] = u32x4{0u, 0u, 0u, 0u};
                if (EXACT || kb * 32 + g * 8 < d) k[x][kb] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + kb * 32));
            }
        }
    };
    u32x4 k[2][KB], qo[KB];
    Pages now = pages(wave), next = pages(wave + WAVES);
    if (wave < n_tiles) {
        request_v(now, wave, 0);
        asm volatile("" ::: "memory");
        request_k(now, wave, k);
    }
    {
        const T* qp = (const T*)q.data + (int64_t)b * q.stride + (int64_t)(h * share + g0 + min(j, nq - 1)) * d + g * 8;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) qo[kb] = EXACT || kb * 32 + g * 8 < d ? *reinterpret_cast<const u32x4*>(qp + kb * 32) : u32x4{0u, 0u, 0u, 0u};
    }
    const float cs = scale * 1.44269504f;
    f32x4 o[OB];
#pragma unroll
    for (int i = 0; i < OB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint32_t read_at[OB];
#pragma unroll
    for (int i = 0; i < OB; ++i) {
        const int row = 4 * g + (j >> 2), pc = i * 2 + ((j & 3) >> 1);
        read_at[i] = lds0 + (row * Ti::CPR + (pc ^ Ti::turn(row))) * 16 + (j & 1) * 8;
    }
    float m = -INFINITY, l = 0.f;
    int buf = 0;
    for (int tile = wave; tile < n_tiles; tile += WAVES) {
        f32x4 s[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                if (EXACT || kb * 32 < d) s[x] = mma16(E{}, k[x][kb], qo[kb], s[x]);
        }
        // K has been waited for just now, and nothing was requested after it: this wait, which V's rows in LDS need, is for nothing more
        asm volatile("" : "+v"(s[0]), "+v"(s[1])::"memory");
        he_bf16::wait_vmcnt<0>();
        const Pages after = pages(tile + 2 * WAVES);
        if (tile + WAVES < n_tiles) {
            request_v(next, tile + WAVES, buf ^ 1);  // (its reads were over when the tile before this one was)
            asm volatile("" ::: "memory");
            request_k(next, tile + WAVES, k);
        }
        const int t0 = begin + tile * 32;
        const int n0 = now.p[0] < 0 ? 0 : min(end - t0, 16), n1 = now.p[1] < 0 ? 0 : min(end - t0 - 16, 16);  // keys of each half
        s[0] *= cs;
        s[1] *= cs;
        if (n0 < 16 || n1 < 16) {
            // rows that do not count may hold anything: no weight, and zeros for it to multiply
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (4 * g + r >= n0) s[0][r] = -INFINITY;
                if (4 * g + r >= n1) s[1][r] = -INFINITY;
            }
#pragma unroll
            for (int n = 0; n < Ti::LOADS; ++n) {
                const int r = n * Ti::RPN + lane / Ti::CPR;
                if ((r & 15) >= (r < 16 ? n0 : n1)) reinterpret_cast<u32x4*>(region + buf * (REGION / 2))[n * 64 + lane] = u32x4{0u, 0u, 0u, 0u};
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int r = 1; r < 8; ++r) top = fmaxf(top, s[r >> 2][r & 3]);
        top = fmaxf(m, lane_max32_apart(lane_max16_apart(top)));
        const float ref = top > -INFINITY ? top : 0.f;
        if (__any(top > m)) {
            const float keep = __builtin_amdgcn_exp2f(m - ref);
            l *= keep;
#pragma unroll
            for (int i = 0; i < OB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] *= keep;
            m = top;
        }
        float w[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) w[r] = __builtin_amdgcn_exp2f(s[r >> 2][r & 3] - ref);
        l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            hi[r] = E::pack(w[2 * r], w[2 * r + 1]);
            lo[r] = E::pack(w[2 * r] - E::lo(hi[r]), w[2 * r + 1] - E::hi(hi[r]));
        }
        const u32x4 wh = {hi[0], hi[1], hi[2], hi[3]}, wl = {lo[0], lo[1], lo[2], lo[3]};
#pragma unroll
        for (int i = 0; i < OB; i += 4) {
            if (!EXACT && i * 16 >= d) continue;
            uint32_t at[4];
            u32x4 v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) at[x] = read_at[i + x] + buf * (REGION / 2);
            v_operands<16 * Ti::CPR * 16>(v, at);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                o[i + x] = mma16(E{}, v[x], wl, o[i + x]);
                o[i + x] = mma16(E{}, v[x], wh, o[i + x]);
            }
        }
        now = next;
        next = after;
        buf ^= 1;
    }
    l = lane_sum32_apart(lane_sum16_apart(l));
    float* mine = reinterpret_cast<float*>(region);
#pragma unroll
    for (int i = 0; i < OB; ++i)
        if (j < nq) *reinterpret_cast<f32x4*>(mine + j * PITCH + i * 16 + 4 * g) = o[i];
    if (g == 0) ml[wave][j] = make_float2(m, l);
    __syncthreads();
    const Partial part_at = partial_of(workspace, (size_t)gridDim.y * n_heads, splits);
    for (int x = threadIdx.x; x < nq * (d / 2); x += 64 * WAVES) {
        const int qi = x / (d / 2), e = x % (d / 2) * 2, head = h * share + g0 + qi;
        float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[w][qi].x);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 a = ml[w][qi], v = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(smem + w * REGION) + qi * PITCH + e);
            const float f = a.x > -INFINITY ? __builtin_amdgcn_exp2f(a.x - top) : a.y;
            sum += a.y * f;
            o0 += v.x * f;
            o1 += v.y * f;
        }
        if (splits == 1) {
            *reinterpret_cast<uint32_t*>((T*)out.data + (int64_t)b * out.stride + (int64_t)head * d + e) = E::pack(attended(sum, o0), attended(sum, o1));
            continue;
        }
        const size_t row = ((size_t)b * n_heads + head) * splits + part;
        if (e == 0) part_at.ml[row] = make_float2(top * 0.693147181f, sum);  // (the join's maxima are natural)
        *reinterpret_cast<float2*>(part_at.o + row * d + e) = make_float2(o0, o1);
    }
}

// The splits of a row, weighted by exp(their maximum - the largest): a split to a lane for the weights, then four dimensions to a thread and the
// splits dealt out to as many groups of threads as there are, whose sums are added in their order.
constexpr int kMostSplits = 64;

template <class E>
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ workspace, Rows out, int n_heads, int d, int splits) {
    typedef typename E::T T;
    __shared__ float weight[kMostSplits];
    __shared__ float4 part[256];
    const int row = blockIdx.x, b = row / n_heads, h = row % n_heads, lane = threadIdx.x & 63;
    const Partial p = partial_of(const_cast<float*>(workspace), gridDim.x, splits);
    const float2 a = lane < splits ? p.ml[(size_t)row * splits + lane] : make_float2(-INFINITY, 0.f);
    const float top = lane_max<64>(a.x);
    const float f = a.y == 0.f ? 0.f : a.x > -INFINITY ? expf(a.x - top) : a.y;  // (a split that saw no key; or a NaN)
    const float l = lane_sum<64>(a.y == 0.f ? 0.f : a.y * f);
    if (threadIdx.x < kMostSplits) weight[threadIdx.x] = f;
    __syncthreads();
    const int lanes = d >> 2, groups = 256 / lanes, e = threadIdx.x % lanes, g = threadIdx.x / lanes;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (g < groups) {
#pragma unroll 4
        for (int s = g; s < splits; s += groups) {
            const float w = weight[s];
            const float4 v = *reinterpret_cast<const float4*>(p.o + ((size_t)row * splits + s) * d + e * 4);
            const bool some = w != 0.f;  // (else what lies there is no one's)
            o.x += some ? v.x * w : 0.f;
            o.y += some ? v.y * w : 0.f;
            o.z += some ? v.z * w : 0.f;
            o.w += some ? v.w * w : 0.f;
        }
    }
    part[threadIdx.x] = o;
    __syncthreads();
    if (g != 0) return;
    for (int x = 1; x < groups; ++x) {
        const float4 v = part[x * lanes + e];
        o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
    }
    T* op = (T*)out.data + (int64_t)b * out.stride + (int64_t)h * d + e * 4;
    const float y0 = attended(l, o.x), y1 = attended(l, o.y), y2 = attended(l, o.z), y3 = attended(l, o.w);
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(op) = make_float4(y0, y1, y2, y3);
    else *reinterpret_cast<uint2*>(op) = make_uint2(E::pack(y0, y1), E::pack(y2, y3));
}

}  // namespace

// Splits of a sequence: enough workgroups for two to a CU (the vector units' kernel: four) as long as each has 128 positions, and up to eight to a CU
// of 1024 positions and more, which even out sequences of different lengths.  us, with 2 / 4 / 8 to a CU: 4 sequences of up to 100003, 40/8 heads
// 195.9 / 200.6 / 187.1; 32 of up to 511, 40/8 heads 17.0 / 19.1 / 19.1; 16 of up to 300, 32 heads of 64 9.7 / 12.7 / 13.0; float, 4 of up to 1000, 32 heads
// 22.1 / 20.8 / 20.6.
int paged_splits(he_dtype dt, int page_size, int n_heads, int n_kv_heads, int n_seqs, int max_len) {
    const bool mma = dt != HE_F32 && page_size >= 16;
    const int share = n_heads / n_kv_heads, per_group = mma ? 16 : 4;
    const int64_t groups = (int64_t)n_seqs * n_kv_heads * ((share + per_group - 1) / per_group), cus = he_bf16::num_cus();
    auto fill = [&](int to_a_cu, int positions) { return std::min<int64_t>((to_a_cu * cus + groups - 1) / groups, (max_len + positions - 1) / positions); };
    return (int)std::min<int64_t>(std::max<int64_t>(std::max(fill(mma ? 2 : 4, 128), fill(8, 1024)), 1), kMostSplits);
}

void paged_attention(hipStream_t s, he_dtype dt, const Cache& c, Rows q, int n_heads, Rows out, const int32_t* lens, int n_seqs, int splits,
                     float scale, float* workspace) {
    const int share = n_heads / c.n_kv_heads;
    by_type(dt, [&](auto e) {
        typedef decltype(e) E;
        if constexpr (sizeof(typename E::T) == 2) {
            if (c.page_shift >= 4) {  // (a half of a tile lies in one page)
                const int groups = c.n_kv_heads * ((share + 15) / 16) * splits;
                auto launch = [&](auto dp, auto exact) {
                    constexpr int DP = decltype(dp)::value;
                    paged_mma_kernel<E, DP, decltype(exact)::value>
                        <<<dim3(groups, n_seqs), 256, 4 * 2 * 32 * DP * 2, s>>>(c, q, n_heads, out, lens, splits, scale, workspace);
                };
                if (c.head_dim == 64) launch(std::integral_constant<int, 64>{}, std::true_type{});
                else if (c.head_dim == 128) launch(std::integral_constant<int, 128>{}, std::true_type{});
                else if (c.head_dim < 128) launch(std::integral_constant<int, 128>{}, std::false_type{});
                else launch(std::integral_constant<int, 256>{}, std::false_type{});
                if (splits > 1) join_kernel<E><<<n_seqs * n_heads, 256, 0, s>>>(workspace, out, n_heads, c.head_dim, splits);
                return;
            }
        }
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
