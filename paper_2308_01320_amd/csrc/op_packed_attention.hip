// Attention over whole prompts laid end to end, on the matrix cores.
//
//   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i),  s_ij = scale q_i . k_j,  m_i = max_j s_ij,  j over i's sequence (up to i)
//
// in one pass over the keys with running m and sum.  A wavefront owns 32 queries of a head, the wavefronts of a workgroup share tiles of
// keys and values through LDS.  Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane owns one query:
// its scores lie in its own accumulators, maximum and sum need one exchange with lane ^ 32, and rescaling is by a scalar of the lane.  The
// keys of a step of O^T are taken in the order in which the accumulators of S^T hold them, so P goes from one product into the next
// without leaving its lane.  V lies in LDS as it does in memory and is transposed by the reads (16-bit types).
//
// m is kept in units of log2, so that a weight is a multiply-add and the hardware's 2^x, and it moves only when a score exceeds it by
// more than 8: weights are then at most 2^8, and most tiles rescale nothing.  Weights of the 16-bit types are rounded once to the type
// (half a step of a weight; a second term costs half as many matrix instructions again), sums are of the unrounded ones.
//
// A row whose result is not finite is summed again over its own keys alone, on the vector units: a weight of nothing times an infinity or a NaN that
// the row does not see must not reach it, and looking for those in the loop would cost every tile.
//
// What bounds it: long prompts, the matrix and vector units in turn (per 64 keys and wavefront 1024 cycles of products, some 950 of soft-max, two
// wavefronts to a SIMD): 8189 tokens, 32/8 heads of 128, bf16 550 us = 1.0 PFLOP/s, where a library's product of 8192^3 reaches 1.22.  Short ones, the
// chain from the sequences' starts over queries and the first tiles: 32 of up to 256, 40 heads 60 us for 214 MB; one of 250 9.9 us.  Float: its
// matrix instructions, a sixteenth of the rate (4 x 700, 8 heads of 64, 45 us).
#include <algorithm>

#include "bf16_common.h"
#include "op_attend.h"

namespace he_op {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// Eight values of a lane as a matrix-core operand: 16 values of k, the lower lanes hold the first eight
template <class E> struct Operand { u32x4 w; };
template <> struct Operand<F32> { float f[8]; };

__device__ __forceinline__ f32x16 mma(const Operand<BF16>& a, const Operand<BF16>& b, f32x16 c) {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a.w), __builtin_bit_cast(v8, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Operand<F16>& a, const Operand<F16>& b, f32x16 c) {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a.w), __builtin_bit_cast(v8, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Operand<F32>& a, const Operand<F32>& b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.f[i], b.f[i], c, 0, 0, 0);  // (k and k + 8 at a time)
    return c;
}

// The tiles: rows of DP values (d rounded up; the pieces past d hold another of the row's, which nothing uses) as 16-byte pieces, piece c of row r at
// place c ^ turn(r): the rows' starts alone would put a column of pieces on few banks.
// SPLIT: the wavefronts of a workgroup have the same queries and 32 keys each of every tile.
template <class E, int DP, int WAVES, bool SPLIT>
struct Tiles {
    typedef typename E::T T;
    static constexpr int N = 16 / sizeof(T), CPR = DP / N;                               // values of a piece, pieces of a row
    static constexpr int BN = SPLIT ? 32 * WAVES : DP * sizeof(T) <= 256 ? 64 : 32;      // keys of a tile
    static constexpr int ROWS = SPLIT ? 32 : 32 * WAVES;                                 // queries of a workgroup
    static constexpr int BYTES = BN * DP * sizeof(T);
    static __device__ __forceinline__ int k_turn(int r) { return CPR >= 16 ? r & 15 : (r >> 1) & 7; }
    // (transposing reads take two pieces of four rows at a time, float reads a row of 32 values)
    static __device__ __forceinline__ int v_turn(int r) { return sizeof(T) == 4 ? 0 : CPR >= 16 ? (r & 7) << 1 : (r & 6); }

    static __device__ __forceinline__ Operand<E> k_operand(const T* lds, int row, int kb, int hh) {
        Operand<E> o;
        if constexpr (sizeof(T) == 2) {
            o.w = *reinterpret_cast<const u32x4*>(lds + (row * CPR + ((kb * 2 + hh) ^ k_turn(row))) * N);
        } else {
            const float4 a = *reinterpret_cast<const float4*>(lds + (row * CPR + ((kb * 4 + hh * 2) ^ k_turn(row))) * N);
            const float4 b = *reinterpret_cast<const float4*>(lds + (row * CPR + ((kb * 4 + hh * 2 + 1) ^ k_turn(row))) * N);
            o.f[0] = a.x; o.f[1] = a.y; o.f[2] = a.z; o.f[3] = a.w; o.f[4] = b.x; o.f[5] = b.y; o.f[6] = b.z; o.f[7] = b.w;
        }
        return o;
    }
    // V^T as operands: dimension block * 32 + lane % 32; keys 16 y + 4 hh + 0..3 and 16 y + 8 + 4 hh + 0..3.  16-bit types: sixteen lanes read
    // four rows of sixteen values, four to a lane, and get a column each.  v_place: where a lane reads for a block, y = 0.
    static __device__ __forceinline__ uint32_t v_place(int block, int lane) {
        const int row = 4 * (lane >> 5) + ((lane & 15) >> 2), c = block * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        return (row * CPR + (c ^ v_turn(row))) * 16 + (lane & 1) * 8;
    }
    // (The compiler puts a wait for the copies in flight ahead of its own transposing reads; these come with the wait for themselves alone.)
    template <int Y>
    static __device__ __forceinline__ void v_operands(Operand<E>* o, const uint32_t (&at)[4]) {
        constexpr int A = Y * 16 * CPR * 16, B = A + 8 * CPR * 16;
        uint2 r[8];
        asm volatile(
            "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
            "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
            "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
            "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
            : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(A), "n"(B)
            : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i].w = u32x4{r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y};
    }
    template <int Y>
    static __device__ __forceinline__ void v_operands(Operand<E>* o, const uint32_t (&at)[2]) {
        constexpr int A = Y * 16 * CPR * 16, B = A + 8 * CPR * 16;
        uint2 r[4];
        asm volatile(
            "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
            "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
            : "v"(at[0]), "v"(at[1]), "n"(A), "n"(B)
            : "memory");
#pragma unroll
        for (int i = 0; i < 2; ++i) o[i].w = u32x4{r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y};
    }
    static __device__ __forceinline__ Operand<E> v_floats(const T* lds, int row0, int block, int lane) {
        Operand<E> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.f[i] = lds[(row0 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3)) * DP + block * 32 + (lane & 31)];
        return o;
    }
};

template <class E>
__device__ __forceinline__ Operand<E> weights8(const float* p) {
    Operand<E> o;
    if constexpr (sizeof(typename E::T) == 2) o.w = u32x4{E::pack(p[0], p[1]), E::pack(p[2], p[3]), E::pack(p[4], p[5]), E::pack(p[6], p[7])};
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) o.f[i] = p[i];
    return o;
}

struct Seq { int begin, end, block; };  // rows of a sequence, and which of its blocks of queries
// The sequence and block of queries that the launch's `at`-th block is: sequences in order, blocks of a sequence last (longest) first.
__device__ __forceinline__ bool block_at(const int32_t* starts, int n_seqs, int n_tokens, int rows, int at, Seq& s) {
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < n_seqs; b0 += 64) {
        const int b = b0 + lane;
        const int begin = b < n_seqs ? min(max(starts[b], 0), n_tokens) : 0, end = b < n_seqs ? min(max(starts[b + 1], begin), n_tokens) : 0;
        const int n = (end - begin + rows - 1) / rows;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            if (lane >= o) upto += x;
        }
        const uint64_t past = __ballot(upto > at);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            s.begin = __builtin_amdgcn_readlane(begin, l);
            s.end = __builtin_amdgcn_readlane(end, l);
            s.block = __builtin_amdgcn_readlane(upto, l) - 1 - at;
            return true;
        }
        at -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

struct PackedArgs {
    Rows q, k, v, out;
    const int32_t* starts;
    int n_heads, n_kv_heads, d, n_seqs, n_tokens, causal;
    float scale;
};

// One query by a wavefront on the vector units, its own keys and no others: where a weight of nothing would meet an infinity or a NaN.
template <class E, int DP>
__device__ __forceinline__ void one_query(const PackedArgs& p, int h, int hk, int row, int begin, int end) {
    typedef typename E::T T;
    constexpr int LPK = DP / 8, KPW = 64 / LPK;
    const int lane = threadIdx.x & 63, sub = lane % LPK;
    float q[8], m = -INFINITY, l = 0.f, acc[8] = {};
    query8<E, DP>((const T*)p.q.data + (int64_t)row * p.q.stride + (int64_t)h * p.d, p.d, p.scale, q);
    for (int j = begin + lane / LPK; j < (end - begin + KPW - 1) / KPW * KPW + begin; j += KPW) {
        const bool ok = j < end;
        Raw8<E> kr = zero8<E>(), vr = zero8<E>();
        if (ok && sub * 8 < p.d) {
            kr = load8<E>((const T*)p.k.data + (int64_t)j * p.k.stride + (int64_t)hk * p.d + sub * 8);
            vr = load8<E>((const T*)p.v.data + (int64_t)j * p.v.stride + (int64_t)hk * p.d + sub * 8);
        }
        float kf[8], vf[8], s = 0.f;
        unpack8<E>(kr, kf);
        unpack8<E>(vr, vf);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(q[e], kf[e], s);
        s = lane_sum<LPK>(s);
        if (!ok) s = -INFINITY;
        const float top = fmaxf(m, s), ref = top > -INFINITY ? top : 0.f, keep = expf(m - ref), w = ok ? expf(s - ref) : 0.f;
        m = top;
        l = l * keep + w;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, vf[e], acc[e] * keep);
    }
    float top = m;
    if (LPK <= 8) top = fmaxf(top, lane_xor8(top));
    if (LPK <= 16) top = lane_max16_apart(top);
    top = lane_max32_apart(top);
    const float own = m > -INFINITY ? expf(m - top) : l, sum = lane_sum_apart<LPK>(l * own);
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = attended(sum, lane_sum_apart<LPK>(acc[e] * own));
    if (lane < LPK && sub * 8 < p.d) store8<E>((T*)p.out.data + (int64_t)row * p.out.stride + (int64_t)h * p.d + sub * 8, pack8<E>(o));
}

// EXACT: the head dimension is DP
template <class E, int DP, bool EXACT, int WAVES, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, !SPLIT && DP * sizeof(typename E::T) <= 256 ? 2 : 1) void packed_attention_kernel(PackedArgs p) {
    typedef typename E::T T;
    typedef Tiles<E, DP, WAVES, SPLIT> Ti;
    constexpr int BN = Ti::BN, SUB = SPLIT ? 1 : BN / 32, KBD = DP / 16, DB = DP / 32, LOADS = BN * Ti::CPR / (64 * WAVES);
    static_assert(LOADS * 64 * WAVES == BN * Ti::CPR, "whole pieces to a thread");
    extern __shared__ __align__(1024) unsigned char smem[];  // two buffers of K and V tiles
    const int d = EXACT ? DP : p.d, share = p.n_heads / p.n_kv_heads;
    // heads that share keys follow each other eight (XCDs) or more apart where there are as many key-value heads, so a key-value head stays in one L2
    const int hq = blockIdx.x % p.n_heads, hk = hq % p.n_kv_heads, h = hk * share + hq / p.n_kv_heads;
    Seq seq;
    if (!block_at(p.starts, p.n_seqs, p.n_tokens, Ti::ROWS, blockIdx.x / p.n_heads, seq)) return;  // (the whole workgroup)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, j = lane & 31, hh = lane >> 5;
    const int q0 = seq.begin + seq.block * Ti::ROWS + (SPLIT ? 0 : wave * 32);  // this wavefront's first query
    const int last_q = min(seq.end, seq.begin + (seq.block + 1) * Ti::ROWS) - 1, sub0 = SPLIT ? wave * 32 : 0;  // ... and its part of a tile
    const int keys = (p.causal ? last_q + 1 : seq.end) - seq.begin, n_tiles = (keys + BN - 1) / BN;
    // the tiles this wavefront takes part in, and the first with keys that some query of it does not see
    const int my_keys = q0 >= seq.end ? 0 : p.causal ? min(q0 + 32, seq.end) - seq.begin : keys;
    const int my_tiles = (my_keys - sub0 + BN - 1) / BN, mask_from = ((p.causal ? q0 - seq.begin + 1 : seq.end - seq.begin) - sub0) / BN;
    const int seen = (p.causal ? min(q0 + j + 1, seq.end) : seq.end) - seq.begin;  // keys this lane's query sees
    // The copies of a tile: piece s of it to lane s % 64; a lane's row moves on by RPN from copy to copy, and the turn of its pieces comes round
    // every PERIOD of them, so that what a copy adds to the lane's offset is the same for all lanes.
    constexpr int RPN = 64 * WAVES / Ti::CPR, PERIOD = RPN >= 16 ? 1 : 16 / RPN < LOADS ? 16 / RPN : LOADS;
    const char* kg = (const char*)p.k.data + ((int64_t)seq.begin * p.k.stride + (int64_t)hk * d) * sizeof(T);
    const char* vg = (const char*)p.v.data + ((int64_t)seq.begin * p.v.stride + (int64_t)hk * d) * sizeof(T);
    const int ks = (int)p.k.stride * (int)sizeof(T), vs = (int)p.v.stride * (int)sizeof(T), r0 = threadIdx.x / Ti::CPR;  // (64 rows of 2^22 values: 2^30)
    uint32_t kc[PERIOD], vc[PERIOD];
#pragma unroll
    for (int n = 0; n < PERIOD; ++n) {
        const int r = r0 + n * RPN, c = threadIdx.x % Ti::CPR;
        int ck = c ^ Ti::k_turn(r), cv = c ^ Ti::v_turn(r);
        if (!EXACT) { ck = min(ck, d / Ti::N - 1); cv = min(cv, d / Ti::N - 1); }
        kc[n] = ck * 16;
        vc[n] = cv * 16;
    }
    const uint32_t k0 = (uint32_t)(r0 * ks), v0 = (uint32_t)(r0 * vs);
    auto stage = [&](int tile, int buf) {
        u32x4* dst = reinterpret_cast<u32x4*>(smem + buf * 2 * Ti::BYTES) + wave * 64;
        const char* kt = kg + (int64_t)tile * BN * ks;
        const char* vt = vg + (int64_t)tile * BN * vs;
        const int left = keys - tile * BN;
        if (left >= BN) {
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                he_bf16::load_block_to_lds(reinterpret_cast<const u32x4*>(kt + (int64_t)n * RPN * ks + (k0 + kc[n % PERIOD])), dst + n * WAVES * 64);
                he_bf16::load_block_to_lds(reinterpret_cast<const u32x4*>(vt + (int64_t)n * RPN * vs + (v0 + vc[n % PERIOD])), dst + Ti::BYTES / 16 + n * WAVES * 64);
            }
        } else {  // behind the last key: the last again, which no query takes from there
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                const int r = min(r0 + n * RPN, left - 1);
                he_bf16::load_block_to_lds(reinterpret_cast<const u32x4*>(kt + ((uint32_t)(r * ks) + kc[n % PERIOD])), dst + n * WAVES * 64);
                he_bf16::load_block_to_lds(reinterpret_cast<const u32x4*>(vt + ((uint32_t)(r * vs) + vc[n % PERIOD])), dst + Ti::BYTES / 16 + n * WAVES * 64);
            }
        }
    };
    stage(0, 0);
    // scores are multiplied by the scale's magnitude; its sign goes into the queries
    const T* qp = (const T*)p.q.data + (int64_t)min(q0 + j, p.n_tokens - 1) * p.q.stride + (int64_t)h * d + hh * 8;
    const uint32_t flip = p.scale < 0.f ? sizeof(T) == 2 ? 0x80008000u : 0x80000000u : 0u;
    auto query = [&](int kb) {
        Operand<E> o;
        if constexpr (sizeof(T) == 2) o.w = *reinterpret_cast<const u32x4*>(qp + kb * 16) ^ flip;
        else {
            float f[8];
            unpack8<E>(load8<E>(qp + kb * 16), f);
#pragma unroll
            for (int e = 0; e < 8; ++e) o.f[e] = __uint_as_float(__float_as_uint(f[e]) ^ flip);
        }
        return o;
    };
    constexpr bool KEEP = DP * sizeof(T) <= 512;  // (float rows of 256: more registers than there are; read again for every tile)
    Operand<E> q[KEEP ? KBD : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int kb = 0; kb < KBD; ++kb)
            if (EXACT || kb * 16 < d) q[kb] = query(kb);
    }
    const float c = fabsf(p.scale) * 1.44269504f;
    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = f32x16{};
    uint32_t v_at[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) v_at[i] = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem + Ti::v_place(i, lane);
    float m = -INFINITY, l = 0.f;
    for (int tile = 0; tile < n_tiles; ++tile) {
        he_bf16::wait_vmcnt<0>();  // this wavefront's copies of the tile
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (tile + 1 < n_tiles) stage(tile + 1, (tile + 1) & 1);  // (everybody has left that buffer)
        if (tile >= my_tiles) continue;                           // (the same for the whole wavefront)
        const T* kt = reinterpret_cast<const T*>(smem + (tile & 1) * 2 * Ti::BYTES);
        const T* vt = reinterpret_cast<const T*>(smem + (tile & 1) * 2 * Ti::BYTES + Ti::BYTES);
        float s[SUB][16];
#pragma unroll
        for (int x = 0; x < SUB; ++x) {
            f32x16 a = f32x16{};
#pragma unroll
            for (int kb = 0; kb < KBD; ++kb) {
                if (EXACT || kb * 16 < d) a = mma(Ti::k_operand(kt, sub0 + x * 32 + j, kb, hh), KEEP ? q[KEEP ? kb : 0] : query(kb), a);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[x][r] = a[r];
        }
        if (tile >= mask_from) {
#pragma unroll
            for (int x = 0; x < SUB; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (tile * BN + sub0 + x * 32 + 8 * (r >> 2) + 4 * hh + (r & 3) >= seen) s[x][r] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int x = 0; x < SUB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[x][r]);
        top = lane_max32_apart(top) * c;
        if (__any(top > m + 8.f)) {
            const float next = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - next);
            m = next;
            l *= keep;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= keep;
        }
#pragma unroll
        for (int x = 0; x < SUB; ++x) {
            float w = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[x][r] = __builtin_amdgcn_exp2f(fmaf(s[x][r], c, -m));
                w += s[x][r];
            }
            l += w;
        }
        if constexpr (sizeof(T) == 2) {
            constexpr int G = DB < 4 ? DB : 4;  // blocks of dimensions whose values are read together
            const uint32_t base = (uint32_t)((tile & 1) * 2 * Ti::BYTES + Ti::BYTES + sub0 * Ti::CPR * 16);
            auto step = [&](auto y) {
                constexpr int Y = decltype(y)::value;
                const Operand<E> w = weights8<E>(&s[Y >> 1][8 * (Y & 1)]);
#pragma unroll
                for (int g = 0; g < DB; g += G) {
                    if (!EXACT && g * 32 >= d) continue;
                    uint32_t at[G];
                    Operand<E> v[G];
#pragma unroll
                    for (int i = 0; i < G; ++i) at[i] = v_at[g + i] + base;
                    Ti::template v_operands<Y>(v, at);
#pragma unroll
                    for (int i = 0; i < G; ++i) o[g + i] = mma(v[i], w, o[g + i]);
                }
            };
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            if constexpr (SUB == 2) {
                step(std::integral_constant<int, 2>{});
                step(std::integral_constant<int, 3>{});
            }
        } else {
#pragma unroll
            for (int y = 0; y < 2 * SUB; ++y) {
                const Operand<E> w = weights8<E>(&s[y >> 1][8 * (y & 1)]);
#pragma unroll
                for (int i = 0; i < DB; ++i)
                    if (EXACT || i * 32 < d) o[i] = mma(Ti::v_floats(vt, sub0 + y * 16, i, lane), w, o[i]);
            }
        }
    }
    l += __shfl_xor(l, 32);
    if constexpr (SPLIT && WAVES > 1) {
        // the wavefronts' parts of the same queries, each on its own scale, added up in their order; a wavefront then has every WAVES-th block of
        // dimensions
        __shared__ float2 ml[WAVES][32];
        __syncthreads();  // (the tiles' memory is free)
        float* parts = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) parts[((wave * DB + i) * 16 + r) * 64 + lane] = o[i][r];
        if (hh == 0) ml[wave][j] = make_float2(m, l);
        __syncthreads();
        float top = -INFINITY, f[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[w][j].x);
        l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 a = ml[w][j];
            f[w] = a.x > -INFINITY ? __builtin_amdgcn_exp2f(a.x - top) : a.y;  // (nothing seen: 0; or a NaN)
            l += a.y * f[w];
        }
#pragma unroll
        for (int i = 0; i < DB; ++i) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v = fmaf(parts[((w * DB + i) * 16 + r) * 64 + lane], f[w], v);
                o[i][r] = v;
            }
        }
    }
    if (q0 >= seq.end) return;
    const float inv = 1.0f / l;
    bool fine = true;
#pragma unroll
    for (int i = 0; i < DB; ++i) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            o[i][r] *= inv;
            fine &= (!EXACT && i * 32 + 8 * (r >> 2) >= d) || fabsf(o[i][r]) < INFINITY;
        }
    }
    const bool mine = q0 + j < seq.end;
    if (__any(mine && !fine)) {  // infinities or NaN among the values: keep what a query does not see out of its sums
        const int n = min(32, seq.end - q0);
        for (int i = SPLIT ? wave : 0; i < n; i += SPLIT ? WAVES : 1) one_query<E, DP>(p, h, hk, q0 + i, seq.begin, p.causal ? q0 + i + 1 : seq.end);
        return;
    }
    T* op = (T*)p.out.data + (int64_t)(mine ? q0 + j : q0) * p.out.stride + (int64_t)h * d;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 8) {
            const int dim = i * 32 + 8 * (r >> 2);  // the lower lanes hold four from here and four from dim + 8, the upper the next four of each
            if ((!EXACT && dim >= d) || (SPLIT && i % WAVES != wave)) continue;
            if constexpr (sizeof(T) == 2) {
                uint32_t a0 = E::pack(o[i][r], o[i][r + 1]), a1 = E::pack(o[i][r + 2], o[i][r + 3]);
                uint32_t b0 = E::pack(o[i][r + 4], o[i][r + 5]), b1 = E::pack(o[i][r + 6], o[i][r + 7]);
                const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
                if (mine) *reinterpret_cast<u32x4*>(op + dim + 8 * hh) = u32x4{(uint32_t)s0[0], (uint32_t)s1[0], (uint32_t)s0[1], (uint32_t)s1[1]};
            } else if (mine) {
                *reinterpret_cast<float4*>(op + dim + 4 * hh) = make_float4(o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]);
                *reinterpret_cast<float4*>(op + dim + 8 + 4 * hh) = make_float4(o[i][r + 4], o[i][r + 5], o[i][r + 6], o[i][r + 7]);
            }
        }
}

}  // namespace

void packed_attention(hipStream_t s, he_dtype dt, Rows q, int n_heads, Rows k, Rows v, int n_kv_heads, int head_dim, Rows out,
                      const int32_t* starts, int n_seqs, int n_tokens, bool causal, float scale) {
    const PackedArgs args{q, k, v, out, starts, n_heads, n_kv_heads, head_dim, n_seqs, n_tokens, causal ? 1 : 0, scale};
    by_type(dt, [&](auto e) {
        typedef decltype(e) E;
        // 128 queries to a workgroup, or 32 whose keys its wavefronts share out: where four times the workgroups fit the CUs at once (float: in three rounds, its
        // products are sixteen times as long against the merge).  us, 128 -> 32 queries: half, 32 heads of 64, 250 tokens 8.5 -> 7.4; bf16,
        // 4 heads of 64, 1500 tokens 26.3 -> 15.2, 8 of 256, 1000 tokens 69.8 -> 45.3, 32 of 128, 250 tokens 11.4 -> 10.6 but 500 tokens
        // 17.2 -> 21.3; float, 8 heads of 64, 2000 tokens 147.7 -> 62.6, 32 of 64, 500 tokens 41.8 -> 26.5.
        auto launch = [&](auto dp, auto exact) {
            constexpr int DP = decltype(dp)::value, TILE = 32 * DP * (int)sizeof(typename E::T) * 4;  // two buffers of 32 keys and values
            constexpr int SHARE = TILE * 4 <= 131072 ? 4 : TILE * 2 <= 131072 ? 2 : 1;
            auto run = [&](auto waves, auto shared) {
                typedef Tiles<E, DP, decltype(waves)::value, decltype(shared)::value> Ti;
                // a sequence has one block more than its rows fill at most
                const unsigned blocks = (unsigned)(n_tokens / Ti::ROWS + std::min(n_seqs, n_tokens));
                packed_attention_kernel<E, DP, decltype(exact)::value, decltype(waves)::value, decltype(shared)::value>
                    <<<blocks * n_heads, 64 * decltype(waves)::value, 4 * Ti::BYTES, s>>>(args);
            };
            if constexpr (SHARE > 1) {  // (a tile of float rows of 256 is as much as LDS holds)
                const int64_t at_once = (int64_t)he_bf16::num_cus() * (163840 / (TILE * SHARE + 1024)) * (sizeof(typename E::T) == 4 ? 3 : 1);
                if ((int64_t)((n_tokens + 127) / 128) * n_heads * 4 <= at_once)
                    return run(std::integral_constant<int, SHARE>{}, std::true_type{});
            }
            run(std::integral_constant<int, 4>{}, std::false_type{});
        };
        if (head_dim == 64) launch(std::integral_constant<int, 64>{}, std::true_type{});
        else if (head_dim == 128) launch(std::integral_constant<int, 128>{}, std::true_type{});
        else if (head_dim < 128) launch(std::integral_constant<int, 128>{}, std::false_type{});
        else launch(std::integral_constant<int, 256>{}, std::false_type{});
    });
}

}  // namespace he_op
