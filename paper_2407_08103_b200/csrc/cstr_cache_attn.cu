// Attention of each row's newest tokens over its own key list, one CTA (or one
// cluster of CTAs, which share the list) per row and key / value head.
//
// Mathematics: one pass over the keys with the running maximum m and sum l of a
// softmax in base 2 (x = q.k * scale * log2 e):
//     m' = max(m, x),  l' = l 2^(m - m') + 2^(x - m'),  o' = o 2^(m - m') + 2^(x - m') v
// Partial (m, l, o) of disjoint key sets combine by the same rule, in any
// grouping; here first over the CTA's warps, then over the cluster's CTAs.
//
// Bound: the keys and values are read once and used by a handful of query rows,
// so the kernel is bound by their bytes.  Hence every warp runs by itself over
// its own chunks of 16 keys, with its own ring of asynchronous copies: no
// barrier in the loop, and copies stay in flight while a chunk is worked on.
// The products run on m16n8k16 matrix instructions: with at most 32 query rows
// per pass they are far from being the limit.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <string.h>

#include "cstr_cache.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kWarps = 4;
constexpr int kStages = 3;
constexpr int kChunk = 16;       // keys per step of a warp
constexpr float kLn2 = 0.693147180559945309f;

struct RowParams {
    const void *q;
    long long q_sb, q_st, q_sh;
    const void *pk, *pv;
    long long pk_st, pk_sh, pv_st, pv_sh;
    const void *ck, *cv;
    long long ck_sb, ck_ss, ck_sh, cv_sb, cv_ss, cv_sh;
    float *weight;
    const int32_t *age, *lens, *pos, *n_query;
    void *out;
    long long o_sb, o_st, o_sh;
    float *lse_out;
    int B, T, Hq, Hk, G, D, cap, P;
    float scale_log2;
    int accumulate;
    int split;           // CTAs of a cluster, sharing one key list
    int score_cap;       // slots per query row whose scores fit in shared memory (0: recompute)
    // parts of the prefix kernel (null: none); see cstr_prefix_plan
    const float4 *part_o;
    const float2 *part_ml;
    int pairs, tiles, grid;
    unsigned long long *oob;
};

// The prefix kernel's parts for one query row: blocks first, first + step, ... (n of them), at `row`.
struct PartList {
    long long first;
    int n, step, row;
};

__device__ __forceinline__ PartList parts_of(const RowParams &p, int kh, int m)
{
    const int pair = m >> 8, local = m & 255;
    const bool two_tiles = p.B * p.G * p.T - (pair << 8) > 128;
    const long long item = (long long)kh * p.pairs + pair, units = (long long)p.Hk * p.pairs * p.tiles;
    const long long c0 = ((item * p.tiles + 1) * p.grid - 1) / units;
    const long long c1 = ((item + 1) * p.tiles * p.grid - 1) / units;
    PartList l;
    l.row = local & 127;
    if (two_tiles) {
        l.first = (c0 + item) * 2 + (local >> 7);
        l.step = 2;
        l.n = (int)(c1 - c0 + 1);
    } else {
        l.first = (c0 + item) * 2;
        l.step = 1;
        l.n = 2 * (int)(c1 - c0 + 1);
    }
    return l;
}

template <typename T> struct Half2;
template <> struct Half2<__nv_bfloat16> {
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<unsigned *>(&v);
    }
    static __device__ __forceinline__ float2 unpack(unsigned u)
    {
        return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&u));
    }
    static __device__ __forceinline__ bool finite(unsigned short h) { return (h & 0x7f80u) != 0x7f80u; }
};
template <> struct Half2<__half> {
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<unsigned *>(&v);
    }
    static __device__ __forceinline__ float2 unpack(unsigned u)
    {
        return __half22float2(*reinterpret_cast<__half2 *>(&u));
    }
    static __device__ __forceinline__ bool finite(unsigned short h) { return (h & 0x7c00u) != 0x7c00u; }
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ unsigned smem_addr(const void *p)
{
    return (unsigned)__cvta_generic_to_shared(p);
}

// 16 bytes to shared memory, or 16 zero bytes where !ok (src is then not read)
__device__ __forceinline__ void copy16(unsigned dst, const void *src, bool ok)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copy4(unsigned dst, const void *src, bool ok)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(ok ? 4 : 0)
                 : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldsm4(unsigned (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(unsigned (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const unsigned (&a)[4], unsigned b0,
                                                        unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
                 "{%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const unsigned (&a)[4], unsigned b0,
                                                 unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
                 "{%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk `ch` of row `r` in a tile of DP-element rows: the
// chunk index is XORed with the row so that the eight rows of an 8x8 matrix hit
// all 32 banks.
template <int DP> __device__ __forceinline__ unsigned tile_off(int r, int ch)
{
    return (unsigned)(r * DP * 2 + ((ch ^ (r & 7)) << 4));
}

template <int DP> struct RowShape {
    static constexpr int kTile = kChunk * DP * 2;                // bytes of one K (or V) chunk
    static constexpr int kStage = 2 * kTile + kChunk * 4;        // K, V, ages
    static constexpr int kRing = kWarps * kStages * kStage;
};

// Key list of one CTA: indices [x0, x1) of the row's list (prefix keys, then slots).
template <typename T, int DP>
struct KeySource {
    const RowParams &p;
    const char *ckb, *cvb, *pkb, *pvb;
    const int32_t *ageb;
    int x0, x1;

    __device__ __forceinline__ void fetch(unsigned stage, int base, int lane, bool want_v) const
    {
        constexpr int CH = DP / 8;                 // 16-byte chunks per key
        constexpr int KPI = 32 / CH;               // keys per warp instruction
        const int ch = lane % CH;
        const bool ch_ok = ch * 8 < p.D;
#pragma unroll
        for (int i = 0; i < kChunk / KPI; ++i) {
            const int key = i * KPI + lane / CH;
            const int x = base + key;
            const bool ok = x < x1 && ch_ok;
            const char *ks, *vs;
            if (x < p.P) {
                ks = pkb + (long long)x * p.pk_st * 2;
                vs = pvb + (long long)x * p.pv_st * 2;
            } else {
                const int j = x - p.P;
                ks = ckb + (long long)j * p.ck_ss * 2;
                vs = cvb + (long long)j * p.cv_ss * 2;
            }
            const unsigned off = tile_off<DP>(key, ch);
            copy16(stage + off, ok ? ks + ch * 16 : ckb, ok);
            if (want_v)
                copy16(stage + RowShape<DP>::kTile + off, ok ? vs + ch * 16 : cvb, ok);
        }
        if (ageb && lane < kChunk) {
            const int j = base + lane - p.P;
            const bool ok = j >= 0 && base + lane < x1;
            copy4(stage + 2 * RowShape<DP>::kTile + lane * 4, ok ? ageb + j : ageb, ok);
        }
    }
};

// x = scaled scores of 16 query rows against the chunk's 16 keys, in the
// accumulator layout: x[n][0..1] = row lane / 4, keys 8 n + 2 (lane % 4) + 0..1;
// x[n][2..3] = row lane / 4 + 8.  Keys a row does not see get -infinity.
template <typename T, int DP>
__device__ __forceinline__ void chunk_scores(float (&x)[2][4], const RowParams &p, unsigned sq,
                                             unsigned stage, int rb, int lane, int base, int x1,
                                             const int (&limit)[2], bool causal)
{
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x[n][e] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        unsigned a[4], b[4];
        ldsm4(a, sq + tile_off<DP>(rb * 16 + (lane & 15), 2 * k + (lane >> 4)));
        // matrices: keys 0-7 / 8-15 x the two 8-element halves of this k step
        ldsm4(b, stage + tile_off<DP>((lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
        mma16816<T>(x[0], a, b[0], b[1]);
        mma16816<T>(x[1], a, b[2], b[3]);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int key = 8 * n + 2 * (lane & 3) + (e & 1);
            bool seen = base + key < x1;
            if (limit[e >> 1] == INT_MIN)          // a query row that does not exist
                seen = false;
            else if (causal && base + key >= p.P) {
                int age;
                asm volatile("ld.shared.s32 %0, [%1];" : "=r"(age)
                             : "r"(stage + 2 * RowShape<DP>::kTile + key * 4) : "memory");
                seen = seen && age <= limit[e >> 1];
            }
            x[n][e] = seen ? x[n][e] * p.scale_log2 : -CUDART_INF_F;
        }
}

// A key that only some query rows see must not reach the others through 0 x NaN:
// where such a key's value row holds something that is not finite, its products
// are added one by one for the rows that see it, and the row is zeroed before
// the matrix product.  At most the row's newest tokens are such keys.
template <typename T, int DP, int RBT>
__device__ __noinline__ void add_nonfinite_values(float (&o)[RBT][DP / 8][4], const float (&x)[RBT][2][4],
                                                  char *vtile, int lane)
{
    unsigned bad = 0;
    for (int i = lane; i < kChunk * DP / 8; i += 32) {
        const int key = i / (DP / 8), ch = i % (DP / 8);
        const uint4 v = *reinterpret_cast<const uint4 *>(vtile + tile_off<DP>(key, ch));
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
        for (int h = 0; h < 4; ++h)
            if (!Half2<T>::finite((unsigned short)w[h]) || !Half2<T>::finite((unsigned short)(w[h] >> 16)))
                bad |= 1u << key;
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    for (; bad; bad &= bad - 1) {
        const int key = __ffs((int)bad) - 1;
        const int src = (lane & ~3) | ((key & 7) >> 1);
#pragma unroll
        for (int rb = 0; rb < RBT; ++rb) {
            const float p0 = __shfl_sync(0xffffffffu, x[rb][0][0], src), p1 = __shfl_sync(0xffffffffu, x[rb][0][1], src);
            const float p2 = __shfl_sync(0xffffffffu, x[rb][1][0], src), p3 = __shfl_sync(0xffffffffu, x[rb][1][1], src);
            const float p4 = __shfl_sync(0xffffffffu, x[rb][0][2], src), p5 = __shfl_sync(0xffffffffu, x[rb][0][3], src);
            const float p6 = __shfl_sync(0xffffffffu, x[rb][1][2], src), p7 = __shfl_sync(0xffffffffu, x[rb][1][3], src);
            const float lo = key < 8 ? (key & 1 ? p1 : p0) : (key & 1 ? p3 : p2);
            const float hi = key < 8 ? (key & 1 ? p5 : p4) : (key & 1 ? p7 : p6);
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
                const unsigned u = *reinterpret_cast<const unsigned *>(vtile + tile_off<DP>(key, n) + (lane & 3) * 4);
                const float2 v = Half2<T>::unpack(u);
                if (lo != 0.f) {
                    o[rb][n][0] += lo * v.x;
                    o[rb][n][1] += lo * v.y;
                }
                if (hi != 0.f) {
                    o[rb][n][2] += hi * v.x;
                    o[rb][n][3] += hi * v.y;
                }
            }
        }
        __syncwarp();
        for (int ch = lane; ch < DP / 8; ch += 32)
            *reinterpret_cast<uint4 *>(vtile + tile_off<DP>(key, ch)) = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
    }
}

template <typename T, int DP, int RBT>
__global__ void __launch_bounds__(kWarps * 32)
row_attention_kernel(const __grid_constant__ RowParams p)
{
    constexpr int ROWS = 16 * RBT;
    using Shape = RowShape<DP>;
    extern __shared__ __align__(128) char smem[];
    char *s_q = smem;                                              // [ROWS][DP] of T
    float *s_stat = reinterpret_cast<float *>(s_q + ROWS * DP * 2); // [2 kWarps + 3][ROWS]
    char *s_ring = reinterpret_cast<char *>(s_stat + (2 * kWarps + 3) * ROWS);
    float *s_o = reinterpret_cast<float *>(s_ring);                // [kWarps][ROWS][DP], after the loop
    constexpr int kArea = Shape::kRing > kWarps * ROWS * DP * 4 ? Shape::kRing : kWarps * ROWS * DP * 4;
    float *s_score = reinterpret_cast<float *>(s_ring + kArea);    // [ROWS][score_cap]
    float *s_m = s_stat, *s_l = s_stat + kWarps * ROWS;            // per warp
    float *s_cm = s_stat + 2 * kWarps * ROWS, *s_cl = s_cm + ROWS, *s_lse = s_cl + ROWS;

    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int item = blockIdx.x / p.split, part = blockIdx.x - item * p.split;
    const int b = item / p.Hk, kh = item - b * p.Hk;
    const int R = p.G * p.T;
    const int len = min(max(p.lens[b], 0), p.cap);
    const int nq = p.n_query ? min(max(p.n_query[b], 0), p.T) : p.T;
    const bool causal = p.pos != nullptr;
    const int pos = causal ? p.pos[b] : 0;

    // this CTA's share of the row's key list, in whole chunks
    const int total = p.P + len;
    const int chunks = (total + kChunk - 1) / kChunk;
    const int per = (chunks + p.split - 1) / p.split;
    KeySource<T, DP> src = {
        p,
        (const char *)p.ck + ((long long)b * p.ck_sb + (long long)kh * p.ck_sh) * 2,
        (const char *)p.cv + ((long long)b * p.cv_sb + (long long)kh * p.cv_sh) * 2,
        (const char *)p.pk + (long long)kh * p.pk_sh * 2,
        (const char *)p.pv + (long long)kh * p.pv_sh * 2,
        causal ? p.age + ((long long)b * p.Hk + kh) * p.cap : nullptr,
        min(part * per * kChunk, total), min((part + 1) * per * kChunk, total)};
    const int n_chunks = (src.x1 - src.x0 + kChunk - 1) / kChunk;
    const int s0 = max(src.x0, p.P), s1 = max(src.x1, p.P);        // own slots: [s0 - P, s1 - P)
    const bool keep = p.accumulate && s1 - s0 <= p.score_cap;
    const unsigned ring = smem_addr(s_ring) + warp * kStages * Shape::kStage;
    const unsigned sq = smem_addr(s_q);

    for (int r0 = 0; r0 < R; r0 += ROWS) {
        const int nr = min(ROWS, R - r0);
        for (int i = tid; i < ROWS * (DP / 8); i += kWarps * 32) {
            const int r = i / (DP / 8), ch = i % (DP / 8);
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (r < nr && ch * 8 < p.D) {
                const int t = (r0 + r) / p.G, g = (r0 + r) - t * p.G;
                const char *s = (const char *)p.q + ((long long)b * p.q_sb + (long long)t * p.q_st +
                                                     (long long)(kh * p.G + g) * p.q_sh) * 2;
                v = *reinterpret_cast<const uint4 *>(s + ch * 16);
            }
            *reinterpret_cast<uint4 *>(s_q + tile_off<DP>(r, ch)) = v;
        }
        __syncthreads();

        // last position that each of this lane's query rows sees
        int limit[RBT][2];
#pragma unroll
        for (int rb = 0; rb < RBT; ++rb)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = rb * 16 + h * 8 + (lane >> 2);
                const int t = (r0 + r) / p.G;
                limit[rb][h] = r < nr && t < nq ? (causal ? pos + t : 0) : INT_MIN;
            }

        float o[RBT][DP / 8][4], m[RBT][2], l[RBT][2];
#pragma unroll
        for (int rb = 0; rb < RBT; ++rb) {
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[rb][n][e] = 0.f;
            m[rb][0] = m[rb][1] = -CUDART_INF_F;
            l[rb][0] = l[rb][1] = 0.f;
        }

#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) {
            const int c = warp + s * kWarps;
            if (c < n_chunks)
                src.fetch(ring + s * Shape::kStage, src.x0 + c * kChunk, lane, true);
            copy_commit();
        }
        int slot = 0;
        for (int c = warp; c < n_chunks; c += kWarps) {
            {
                const int ahead = c + (kStages - 1) * kWarps;
                const int into = slot == 0 ? kStages - 1 : slot - 1;
                if (ahead < n_chunks)
                    src.fetch(ring + into * Shape::kStage, src.x0 + ahead * kChunk, lane, true);
                copy_commit();
            }
            copy_wait<kStages - 1>();
            __syncwarp();
            const unsigned stage = ring + slot * Shape::kStage;
            const int base = src.x0 + c * kChunk;
            float x[RBT][2][4];
#pragma unroll
            for (int rb = 0; rb < RBT; ++rb)
                chunk_scores<T, DP>(x[rb], p, sq, stage, rb, lane, base, src.x1, limit[rb], causal);
            if (keep) {
#pragma unroll
                for (int rb = 0; rb < RBT; ++rb)
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int r = rb * 16 + (e >> 1) * 8 + (lane >> 2);
                            const int at = base + 8 * n + 2 * (lane & 3) + (e & 1);
                            if (r < nr && at >= s0 && at < s1)
                                s_score[r * p.score_cap + at - s0] = x[rb][n][e];
                        }
            }
            bool some = false;                       // a key seen by some rows of the call only
            if (causal && p.T > 1 && lane < kChunk && base + lane >= p.P && base + lane < src.x1) {
                int age;
                asm volatile("ld.shared.s32 %0, [%1];" : "=r"(age)
                             : "r"(stage + 2 * Shape::kTile + lane * 4) : "memory");
                some = age > pos;
            }
            const bool partial = __any_sync(0xffffffffu, some);
#pragma unroll
            for (int rb = 0; rb < RBT; ++rb) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = fmaxf(fmaxf(x[rb][0][2 * h], x[rb][0][2 * h + 1]),
                                      fmaxf(x[rb][1][2 * h], x[rb][1][2 * h + 1]));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const float mn = fmaxf(m[rb][h], top);
                    const float ref = mn == -CUDART_INF_F ? 0.f : mn;
                    const float f = exp2_fast(m[rb][h] - ref);
                    m[rb][h] = mn;
                    float sum = 0.f;
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float &v = x[rb][n][2 * h + e];
                            v = exp2_fast(v - ref);
                            sum += v;
                        }
                    l[rb][h] = l[rb][h] * f + sum;
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n) {
                        o[rb][n][2 * h] *= f;
                        o[rb][n][2 * h + 1] *= f;
                    }
                }
            }
            if (partial)
                add_nonfinite_values<T, DP, RBT>(o, x, s_ring + (warp * kStages + slot) * Shape::kStage + Shape::kTile, lane);
            // the probabilities enter the second product in the values' type: rounded to nearest,
            // like the values themselves; the sum l keeps the unrounded ones
            unsigned a[RBT][4];
#pragma unroll
            for (int rb = 0; rb < RBT; ++rb) {
                a[rb][0] = Half2<T>::pack(x[rb][0][0], x[rb][0][1]);
                a[rb][1] = Half2<T>::pack(x[rb][0][2], x[rb][0][3]);
                a[rb][2] = Half2<T>::pack(x[rb][1][0], x[rb][1][1]);
                a[rb][3] = Half2<T>::pack(x[rb][1][2], x[rb][1][3]);
            }
#pragma unroll
            for (int n2 = 0; n2 < DP / 16; ++n2) {
                unsigned v[4];
                ldsm4_trans(v, stage + Shape::kTile + tile_off<DP>(lane & 15, 2 * n2 + (lane >> 4)));
#pragma unroll
                for (int rb = 0; rb < RBT; ++rb) {
                    mma16816<T>(o[rb][2 * n2], a[rb], v[0], v[1]);
                    mma16816<T>(o[rb][2 * n2 + 1], a[rb], v[2], v[3]);
                }
            }
            __syncwarp();
            slot = slot + 1 == kStages ? 0 : slot + 1;
        }
        copy_wait<0>();

        // the warps' partial results meet in shared memory (the ring is free by now)
        __syncthreads();
#pragma unroll
        for (int rb = 0; rb < RBT; ++rb) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = rb * 16 + h * 8 + (lane >> 2);
                float sum = l[rb][h];
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if ((lane & 3) == 0) {
                    s_m[warp * ROWS + r] = m[rb][h];
                    s_l[warp * ROWS + r] = sum;
                }
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
                    *reinterpret_cast<float2 *>(s_o + (warp * ROWS + r) * DP + n * 8 + 2 * (lane & 3)) =
                        make_float2(o[rb][n][2 * h], o[rb][n][2 * h + 1]);
            }
        }
        __syncthreads();
        for (int r = tid; r < nr; r += kWarps * 32) {
            float top = s_m[r];
#pragma unroll
            for (int w = 1; w < kWarps; ++w)
                top = fmaxf(top, s_m[w * ROWS + r]);
            const float ref = top == -CUDART_INF_F ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                // -1: the warp saw no key of this row; whatever its sums hold does not count
                const bool none = s_m[w * ROWS + r] == -CUDART_INF_F;
                const float f = exp2_fast(s_m[w * ROWS + r] - ref);
                sum += f * s_l[w * ROWS + r];
                s_m[w * ROWS + r] = none ? -1.f : f;
            }
            s_cm[r] = top;
            s_cl[r] = sum;
        }
        __syncthreads();
        for (int i = tid; i < nr * (DP / 2); i += kWarps * 32) {
            const int r = i / (DP / 2), d = 2 * (i % (DP / 2));
            float2 v = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = s_m[w * ROWS + r];
                const float2 u = *reinterpret_cast<const float2 *>(s_o + (w * ROWS + r) * DP + d);
                if (f >= 0.f || f != f) {
                    v.x += f * u.x;
                    v.y += f * u.y;
                }
            }
            *reinterpret_cast<float2 *>(s_o + r * DP + d) = v;
        }
        if (p.split > 1)
            cluster.sync();
        else
            __syncthreads();
        if (p.part_ml)
            asm volatile("griddepcontrol.wait;" ::: "memory");      // the prefix kernel has finished

        // ... and the cluster's, through distributed shared memory; each CTA finishes a share
        // of the outputs and the weights of its own slots
        for (int r = tid; r < nr; r += kWarps * 32) {
            float top = -CUDART_INF_F;
            for (int c = 0; c < p.split; ++c)
                top = fmaxf(top, p.split > 1 ? *cluster.map_shared_rank(s_cm + r, c) : s_cm[r]);
            const int t = (r0 + r) / p.G, g = (r0 + r) - t * p.G;
            const bool real = t < nq;
            const PartList parts = p.part_ml && real ? parts_of(p, kh, b * R + r0 + r) : PartList{0, 0, 0, 0};
            for (int i = 0; i < parts.n; ++i)
                top = fmaxf(top, p.part_ml[(parts.first + (long long)i * parts.step) * 128 + parts.row].x);
            const float ref = top == -CUDART_INF_F ? 0.f : top;
            float sum = 0.f;
            for (int i = 0; i < parts.n; ++i) {
                const float2 ml = p.part_ml[(parts.first + (long long)i * parts.step) * 128 + parts.row];
                sum += exp2_fast(ml.x - ref) * ml.y;
            }
            for (int c = 0; c < p.split; ++c)
                sum += p.split > 1 ? exp2_fast(*cluster.map_shared_rank(s_cm + r, c) - ref) * *cluster.map_shared_rank(s_cl + r, c)
                                   : exp2_fast(s_cm[r] - ref) * s_cl[r];
            // nothing seen: +infinity, so that 2^(x - lse) is 0 for every key
            const float lse = sum == 0.f ? CUDART_INF_F : ref + log2f(sum);
            s_lse[r] = lse;
            if (part == 0 && p.lse_out)
                p.lse_out[((long long)b * p.T + t) * p.Hq + kh * p.G + g] =
                    sum == 0.f ? -CUDART_INF_F : lse * kLn2;
        }
        __syncthreads();
        // rows run fastest: the parts keep neighbouring rows side by side
        const int pieces = nr * (p.D / 4);
        for (int i = part * kWarps * 32 + tid; i < pieces; i += p.split * kWarps * 32) {
            const int d4 = i / nr, r = i - d4 * nr;
            const int t = (r0 + r) / p.G, g = (r0 + r) - t * p.G;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add = [&](float m, const float4 &u) {
                const float f = exp2_fast(m - s_lse[r]);
                if (m != -CUDART_INF_F) {
                    v.x += f * u.x;
                    v.y += f * u.y;
                    v.z += f * u.z;
                    v.w += f * u.w;
                }
            };
            if (p.part_ml && t < nq) {
                const PartList parts = parts_of(p, kh, b * R + r0 + r);
                for (int k = 0; k < parts.n; ++k) {
                    const long long block = parts.first + (long long)k * parts.step;
                    const float m = p.part_ml[block * 128 + parts.row].x;
                    // (a part without keys has no outputs)
                    if (m != -CUDART_INF_F)
                        add(m, p.part_o[(block * (DP / 4) + d4) * 128 + parts.row]);
                }
            }
            for (int c = 0; c < p.split; ++c) {
                const float *so = p.split > 1 ? cluster.map_shared_rank(s_o, c) : s_o;
                const float m = p.split > 1 ? *cluster.map_shared_rank(s_cm + r, c) : s_cm[r];
                add(m, *reinterpret_cast<const float4 *>(so + r * DP + 4 * d4));
            }
            char *dst = (char *)p.out + ((long long)b * p.o_sb + (long long)t * p.o_st +
                                         (long long)(kh * p.G + g) * p.o_sh + 4 * d4) * 2;
            *reinterpret_cast<uint2 *>(dst) = make_uint2(Half2<T>::pack(v.x, v.y), Half2<T>::pack(v.z, v.w));
        }
        // the next rows reuse the memory that peers read, and a CTA must not leave while they do.
        // (Every CTA of the cluster takes the same number of cluster barriers: what follows has none.)
        if (p.split > 1)
            cluster.sync();
        else
            __syncthreads();
        if (p.accumulate) {
            float *wrow = p.weight + ((long long)b * p.Hk + kh) * p.cap;
            if (keep) {
                for (int j = tid; j < s1 - s0; j += kWarps * 32) {
                    float w = 0.f;
                    for (int r = 0; r < nr; ++r)
                        w += exp2_fast(s_score[r * p.score_cap + j] - s_lse[r]);
                    const long long at = s0 - p.P + j;
                    if (CSTR_INB(p.oob, at, p.cap, CSTR_SITE_CACHE))
                        wrow[at] += w;
                }
            } else {                                // scores once more from the keys
                float lse[RBT][2];
#pragma unroll
                for (int rb = 0; rb < RBT; ++rb)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = rb * 16 + h * 8 + (lane >> 2);
                        lse[rb][h] = r < nr ? s_lse[r] : CUDART_INF_F;
                    }
                const int first = (s0 - src.x0) / kChunk;
                for (int c = first + warp; c < n_chunks; c += kWarps) {
                    const int base = src.x0 + c * kChunk;
                    src.fetch(ring, base, lane, false);
                    copy_commit();
                    copy_wait<0>();
                    __syncwarp();
                    float w[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
                    for (int rb = 0; rb < RBT; ++rb) {
                        float x[2][4];
                        chunk_scores<T, DP>(x, p, sq, ring, rb, lane, base, src.x1, limit[rb], causal);
#pragma unroll
                        for (int n = 0; n < 2; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                w[n][e & 1] += exp2_fast(x[n][e] - lse[rb][e >> 1]);
                    }
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1)
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            w[n][0] += __shfl_xor_sync(0xffffffffu, w[n][0], off);
                            w[n][1] += __shfl_xor_sync(0xffffffffu, w[n][1], off);
                        }
                    if (lane < 4) {
#pragma unroll
                        for (int n = 0; n < 2; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int at = base + 8 * n + 2 * lane + e;
                                if (at >= s0 && at < s1 &&
                                    CSTR_INB(p.oob, at - p.P, p.cap, CSTR_SITE_CACHE))
                                    wrow[at - p.P] += w[n][e];
                            }
                    }
                    __syncwarp();
                }
            }
        }
        __syncthreads();
    }
}

template <typename T, int DP, int RBT>
int launch(const cstr_cache &c, RowParams p, cudaStream_t stream)
{
    using Shape = RowShape<DP>;
    constexpr int ROWS = 16 * RBT;
    const int area = Shape::kRing > kWarps * ROWS * DP * 4 ? Shape::kRing : kWarps * ROWS * DP * 4;
    const int fixed = ROWS * DP * 2 + (2 * kWarps + 3) * ROWS * 4 + area;
    int smem = fixed;
    p.score_cap = 0;
    if (p.accumulate) {
        const int rows = p.G * p.T < ROWS ? p.G * p.T : ROWS;
        // own slots, at most: a CTA's share of the list may be slots alone
        const long long share = ((long long)p.P + p.cap + p.split - 1) / p.split + kChunk;
        const long long want = share < p.cap ? share : p.cap;
        if (fixed + want * rows * 4 <= 220 * 1024) {
            p.score_cap = (int)want;
            smem += (int)(want * rows * 4);
        }
    }
    auto kernel = row_attention_kernel<T, DP, RBT>;
    CSTR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)((long long)p.B * p.Hk * p.split));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (p.part_ml) {                     // may start beside the prefix kernel, and waits for its parts
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.numAttrs = 2;
    }
    CSTR_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p));
    return CSTR_OK;
}

template <typename T>
int launch_typed(const cstr_cache &c, const RowParams &p, cudaStream_t stream)
{
    const bool wide = c.head_dim > 64;
    // more than 16 query rows: two blocks of 16 per pass, so that the keys are read half as often
    if (p.G * p.T > 16)
        return wide ? launch<T, 128, 2>(c, p, stream) : launch<T, 64, 2>(c, p, stream);
    return wide ? launch<T, 128, 1>(c, p, stream) : launch<T, 64, 1>(c, p, stream);
}

}  // namespace

int cstr_launch_row_attention(const cstr_cache &c, const cstr_row_args &a, bool with_prefix,
                              cudaStream_t stream)
{
    RowParams p;
    memset(&p, 0, sizeof p);
    p.q = a.q;
    p.q_sb = a.q_sb, p.q_st = a.q_st, p.q_sh = a.q_sh;
    p.pk = c.prefix_k, p.pv = c.prefix_v;
    p.pk_st = c.pk_st, p.pk_sh = c.pk_sh, p.pv_st = c.pv_st, p.pv_sh = c.pv_sh;
    p.ck = c.cache_k, p.cv = c.cache_v;
    p.ck_sb = c.ck_sb, p.ck_ss = c.ck_ss, p.ck_sh = c.ck_sh;
    p.cv_sb = c.cv_sb, p.cv_ss = c.cv_ss, p.cv_sh = c.cv_sh;
    p.weight = c.weight;
    p.age = c.age;
    p.lens = c.lens;
    p.pos = a.pos;
    p.n_query = a.n_query;
    p.out = a.out;
    p.o_sb = a.o_sb, p.o_st = a.o_st, p.o_sh = a.o_sh;
    p.lse_out = a.lse_out;
    p.B = c.batch;
    p.T = a.tokens;
    p.Hq = c.n_heads;
    p.Hk = c.n_kv_heads;
    p.G = c.n_heads / c.n_kv_heads;
    p.D = c.head_dim;
    p.cap = c.cap;
    p.P = with_prefix ? (int)c.prefix_len : 0;
    if (!with_prefix) {
        const cstr_prefix_plan s = cstr_plan_prefix(c, a.tokens);
        p.part_o = (const float4 *)c.part_o;
        p.part_ml = (const float2 *)c.part_ml;
        p.pairs = s.pairs;
        p.tiles = s.tiles;
        p.grid = s.grid;
    }
    p.scale_log2 = a.scale_log2;
    p.accumulate = a.accumulate;
    p.oob = CSTR_OOB_RECORD();
    // share a row's keys among CTAs until there are two per SM, or 64 keys a CTA
    const long long items = (long long)p.B * p.Hk;
    p.split = 1;
    while (p.split < 8 && items * p.split < 2LL * c.sm_count &&
           (long long)p.P + p.cap >= 2LL * p.split * 64)
        p.split *= 2;
    if (items * p.split > 0x7fffffffLL)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_cache_attention: batch x heads too large for one launch");
    return c.dtype == CSTR_BF16 ? launch_typed<__nv_bfloat16>(c, p, stream)
                                : launch_typed<__half>(c, p, stream);
}
