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
// The products run on m16n8k16 matrix instructions in transposed form, S' = K Q'
// and O' = V' P': the keys and the head's elements fill the 16 rows of an
// instruction, and its 8 columns are query rows, so that the usual 4 or 8 query
// rows of a key / value head waste nothing (the other way round they would fill
// a quarter or a half of 16).
//
// Measured: 512 rows x 8 heads of up to 1,024 slots, head_dim 128, bf16, weights added
// up, behind 128 prompt tokens: 256 us for 1.64 GB, 6.4 TB/s; behind 16,384 tokens it
// joins the prefix kernel's parts as well (380 - 388 us together, of them 139 the prefix
// kernel's).  Where ages decide what a token sees, looking for slots it does not see
// costs 2.5 us of 269.  Few rows: bound by one CTA's chain of chunks, hence the split.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <string.h>

#include "cstr_cache.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kWarps = 4;
constexpr int kChunk = 16;       // keys per step of a warp
constexpr int kMostSmem = 220 * 1024;   // dynamic shared memory of a CTA, the scores it keeps included
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
    int pairs, tiles, grid, max_parts;
    int narrow;          // units x grid fits in 32 bits
    cstr_divisor by_g;
    unsigned long long *oob;
};

// The prefix kernel's parts for one query row: blocks first, first + 2, ... (n of them), at `row`.
struct PartList {
    int first, n, row;
};

__device__ __forceinline__ PartList parts_of(const RowParams &p, int kh, int m)
{
    const int pair = m >> 8, local = m & 255;
    const int item = kh * p.pairs + pair;
    int c0, c1;                          // first and last CTA with a segment of this row group
    if (p.narrow) {
        const unsigned units = (unsigned)(p.Hk * p.pairs * p.tiles), first = (unsigned)(item * p.tiles);
        c0 = (int)(((first + 1) * p.grid - 1) / units);
        c1 = (int)(((first + p.tiles) * p.grid - 1) / units);
    } else {
        const long long units = (long long)p.Hk * p.pairs * p.tiles, first = (long long)item * p.tiles;
        c0 = (int)(((first + 1) * p.grid - 1) / units);
        c1 = (int)(((first + p.tiles) * p.grid - 1) / units);
    }
    PartList l;
    l.row = local & 127;
    l.first = (c0 + item) * 2 + (local >> 7);
    l.n = c1 - c0 + 1;
    return l;
}

template <typename T> struct Half2;
template <> struct Half2<__nv_bfloat16> {
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<unsigned *>(&v);
    }
    static __device__ __forceinline__ float value(unsigned short h) { return __uint_as_float((unsigned)h << 16); }
    static __device__ __forceinline__ bool finite(unsigned short h) { return (h & 0x7f80u) != 0x7f80u; }
};
template <> struct Half2<__half> {
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<unsigned *>(&v);
    }
    static __device__ __forceinline__ float value(unsigned short h) { return __half2float(__ushort_as_half(h)); }
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

// 8x8 matrix of 16-bit elements, transposed across the warp
__device__ __forceinline__ unsigned transpose8(unsigned v)
{
    unsigned r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
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

// *p += v without waiting for the old value.  Every weight gets exactly one addition per pass,
// always from the CTA that owns the slot, so the result does not depend on any order.
__device__ __forceinline__ void add_once(float *p, float v)
{
    asm volatile("red.global.add.f32 [%0], %1;" ::"l"(p), "f"(v) : "memory");
}

// Byte offset of 16-byte chunk `ch` of row `r` in a tile of DP-element rows: the
// chunk index is XORed with the row so that the eight rows of an 8x8 matrix hit
// all 32 banks.
template <int DP> __device__ __forceinline__ unsigned tile_off(int r, int ch)
{
    return (unsigned)(r * DP * 2 + ((ch ^ (r & 7)) << 4));
}

// kSlots: units (keys or values of a chunk) in a warp's ring.  Two for few query rows of wide heads (512
// rows of 1,024 slots, head_dim 128: 380 us, with three 385 us, with four 486 us);
// three where a unit is half as large (head_dim 64: 265 us, with two 275 us) or is worked on for longer
// (64 rows x 20 query rows: 88.7 us, with two 90.5 us).
template <int DP, int NT> struct RowShape {
    static constexpr int kSlots = DP == 128 && NT == 1 ? 2 : 3;
    static constexpr int kUnit = kChunk * DP * 2 + kChunk * 4;   // keys (or values) of a chunk, ages
    static constexpr int kRing = kWarps * kSlots * kUnit;
    static constexpr int kPitch = DP + 4;                        // floats per row of the partial outputs
};

// Key list of one CTA: indices [x0, x1) of the row's list (prefix keys, then slots).
template <typename T, int DP>
struct KeySource {
    const RowParams &p;
    const char *ckb, *cvb, *pkb, *pvb;
    const int32_t *ageb;
    int x0, x1;

    // the keys (and ages) or the values of the chunk at `base` into a ring slot
    __device__ __forceinline__ void fetch(unsigned to, bool values, int base, int lane) const
    {
        constexpr int CH = DP / 8;                 // 16-byte pieces per key
        constexpr int KPI = 32 / CH;               // keys per warp instruction
        const int ch = lane % CH, key0 = lane / CH;
        const char *slots = values ? cvb : ckb;
        const long long ss = 2 * (values ? p.cv_ss : p.ck_ss);
        if (base >= p.P && base + kChunk <= x1 && DP == p.D) {          // whole chunk of slots
            const char *from = slots + (base - p.P + key0) * ss + ch * 16;
#pragma unroll
            for (int i = 0; i < kChunk / KPI; ++i) {
                copy16(to + tile_off<DP>(i * KPI + key0, ch), from, true);
                from += KPI * ss;
            }
        } else {
            const char *prompt = values ? pvb : pkb;
            const long long st = 2 * (values ? p.pv_st : p.pk_st);
            const bool ch_ok = ch * 8 < p.D;
#pragma unroll 2
            for (int i = 0; i < kChunk / KPI; ++i) {
                const int key = i * KPI + key0;
                const int x = base + key;
                const bool ok = x < x1 && ch_ok;
                const char *from = x < p.P ? prompt + x * st : slots + (x - p.P) * ss;
                copy16(to + tile_off<DP>(key, ch), ok ? from + ch * 16 : slots, ok);
            }
        }
        if (!values && ageb && lane < kChunk) {
            const int j = base + lane - p.P;
            const bool ok = j >= 0 && base + lane < x1;
            copy4(to + kChunk * DP * 2 + lane * 4, ok ? ageb + j : ageb, ok);
        }
    }
};

// Query rows as the second operand of S' = K Q': fragments of k steps k and k + 1.
template <int DP> __device__ __forceinline__ void query_pair(unsigned (&f)[4], unsigned sq, int n, int k, int lane)
{
    ldsm4(f, sq + tile_off<DP>(8 * n + (lane & 7), 2 * k + (lane >> 3)));
}

// x = scaled scores of the chunk's 16 keys against 8 NT query rows, in the accumulator layout:
// x[n][0..1] = key lane / 4, rows 8 n + 2 (lane % 4) + 0..1; x[n][2..3] = key lane / 4 + 8.
// `masked`: -infinity for keys past the list's end and, with `causal`, for slots younger than a
// row's limit.
template <typename T, int DP, int NT>
__device__ __forceinline__ void chunk_scores(float (&x)[NT][4], const RowParams &p, const unsigned (&qf)[NT <= 2 ? NT : 1][DP / 16][2],
                                             unsigned sq, unsigned keys, int lane, int base, int x1, const int (&limit)[NT][2],
                                             bool masked, bool causal)
{
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x[n][e] = 0.f;
    float y[NT][4];                                // odd k steps, so that the chains are half as long
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[n][e] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; k += 2) {
        unsigned a[4], a2[4];
        ldsm4(a, keys + tile_off<DP>(lane & 15, 2 * k + (lane >> 4)));
        ldsm4(a2, keys + tile_off<DP>(lane & 15, 2 * k + 2 + (lane >> 4)));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (NT <= 2) {                         // (constant indices: qf has NT blocks then)
                mma16816<T>(x[n], a, qf[NT <= 2 ? n : 0][k][0], qf[NT <= 2 ? n : 0][k][1]);
                mma16816<T>(y[n], a2, qf[NT <= 2 ? n : 0][k + 1][0], qf[NT <= 2 ? n : 0][k + 1][1]);
            } else {                               // too many to keep in registers
                unsigned f[4];
                query_pair<DP>(f, sq, n, k, lane);
                mma16816<T>(x[n], a, f[0], f[1]);
                mma16816<T>(y[n], a2, f[2], f[3]);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x[n][e] = (x[n][e] + y[n][e]) * p.scale_log2;
    if (!masked)
        return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int key = 8 * h + (lane >> 2);
        int age = INT_MIN;
        if (causal && base + key >= p.P)
            asm volatile("ld.shared.s32 %0, [%1];" : "=r"(age) : "r"(keys + kChunk * DP * 2 + key * 4) : "memory");
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (base + key >= x1 || (causal && age > limit[n][e]))
                    x[n][2 * h + e] = -CUDART_INF_F;
    }
}

// A key that only some query rows see, or none, must not reach the others through
// 0 x NaN: where such a key's value row holds something that is not finite, its
// products are added one by one for the rows that see it, and the row is zeroed
// before the matrix product.  The row's newest tokens are such keys, and with a
// single token every slot that is younger than it.
// (Inlined: the accumulators must not have an address, or they live in memory.)
template <typename T, int DP, int NT>
__device__ __forceinline__ void add_nonfinite_values(float (&o)[NT][DP / 16][4], const float (&x)[NT][4], char *vtile,
                                                     int lane)
{
    unsigned bad = 0;
#pragma unroll 1
    for (int i = lane; i < kChunk * DP / 8; i += 32) {
        const int key = i / (DP / 8), ch = i % (DP / 8);
        const uint4 v = *reinterpret_cast<const uint4 *>(vtile + tile_off<DP>(key, ch));
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
        for (int h = 0; h < 4; ++h)
            if (!Half2<T>::finite((unsigned short)w[h]) || !Half2<T>::finite((unsigned short)(w[h] >> 16)))
                bad |= 1u << key;
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
#pragma unroll 1
    for (; bad; bad &= bad - 1) {
        const int key = __ffs((int)bad) - 1;
        const int src = ((key & 7) << 2) | (lane & 3);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float a0 = __shfl_sync(0xffffffffu, x[n][0], src), a1 = __shfl_sync(0xffffffffu, x[n][1], src);
            const float b0 = __shfl_sync(0xffffffffu, x[n][2], src), b1 = __shfl_sync(0xffffffffu, x[n][3], src);
            const float p0 = key < 8 ? a0 : b0, p1 = key < 8 ? a1 : b1;
#pragma unroll
            for (int j = 0; j < DP / 16; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int d = 16 * j + 8 * h + (lane >> 2);
                    const float v = Half2<T>::value(*reinterpret_cast<const unsigned short *>(
                        vtile + tile_off<DP>(key, d >> 3) + (d & 7) * 2));
                    if (p0 != 0.f)
                        o[n][j][2 * h] += p0 * v;
                    if (p1 != 0.f)
                        o[n][j][2 * h + 1] += p1 * v;
                }
        }
        __syncwarp();
        for (int ch = lane; ch < DP / 8; ch += 32)
            *reinterpret_cast<uint4 *>(vtile + tile_off<DP>(key, ch)) = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
    }
}

// NT: blocks of 8 query rows per pass
template <typename T, int DP, int NT>
__global__ void __launch_bounds__(kWarps * 32, NT == 1 ? 4 : 2)
row_attention_kernel(const __grid_constant__ RowParams p)
{
    constexpr int ROWS = 8 * NT;
    using Shape = RowShape<DP, NT>;
    using Ref = cstr_softmax_reference<T>;
    constexpr int kSlots = Shape::kSlots;
    extern __shared__ __align__(128) char smem[];
    char *s_q = smem;                                              // [ROWS][DP] of T
    float *s_stat = reinterpret_cast<float *>(s_q + ROWS * DP * 2); // [2 kWarps + 3][ROWS]
    char *s_ring = reinterpret_cast<char *>(s_stat + (2 * kWarps + 3) * ROWS);
    float *s_o = reinterpret_cast<float *>(s_ring);                // [kWarps][ROWS][kPitch], after the loop
    constexpr int kOut = kWarps * ROWS * Shape::kPitch * 4;
    constexpr int kArea = Shape::kRing > kOut ? Shape::kRing : kOut;
    float *s_fac = reinterpret_cast<float *>(s_ring + kArea);      // [rows of a pass][max_parts]
    float *s_score = s_fac + min(ROWS, p.G * p.T) * p.max_parts;   // [rows of a pass][score_cap]
    __shared__ PartList s_parts[ROWS];
    float *s_m = s_stat, *s_l = s_stat + kWarps * ROWS;            // per warp
    float *s_cm = s_stat + 2 * kWarps * ROWS, *s_cl = s_cm + ROWS, *s_lse = s_cl + ROWS;

    if (!p.part_ml) {                              // (else the prefix kernel has waited)
        cstr_wait_for_earlier_kernels();
        cstr_let_next_kernel_start();
    }
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
    // scores are kept from the chunk on in which the slots begin
    const int kept0 = (s0 - src.x0) / kChunk * kChunk;
    const bool keep = p.accumulate && n_chunks * kChunk - kept0 <= p.score_cap;
    const int mine = n_chunks > warp ? (n_chunks - warp + kWarps - 1) / kWarps : 0;   // chunks of this warp
    char *ring_ptr = s_ring + warp * kSlots * Shape::kUnit;
    const unsigned ring = smem_addr(ring_ptr);

    for (int r0 = 0; r0 < R; r0 += ROWS) {
        const int nr = min(ROWS, R - r0);
        // the queries and the first chunks are on their way together; unit 2 i is the keys of the
        // warp's chunk i, unit 2 i + 1 its values
        constexpr int kQ = (ROWS * (DP / 8) + kWarps * 32 - 1) / (kWarps * 32);
        uint4 qv[kQ];
#pragma unroll
        for (int k = 0; k < kQ; ++k) {
            const int i = tid + k * kWarps * 32, r = i / (DP / 8), ch = i % (DP / 8);
            qv[k] = make_uint4(0u, 0u, 0u, 0u);
            if (r < nr && ch * 8 < p.D) {
                const int t = p.by_g(r0 + r), g = (r0 + r) - t * p.G;
                const char *s = (const char *)p.q + ((long long)b * p.q_sb + (long long)t * p.q_st +
                                                     (long long)(kh * p.G + g) * p.q_sh) * 2;
                qv[k] = *reinterpret_cast<const uint4 *>(s + ch * 16);
            }
        }
        auto fetch = [&](int unit, int slot) {
            if (unit < 2 * mine)
                src.fetch(ring + slot * Shape::kUnit, unit & 1, src.x0 + ((unit >> 1) * kWarps + warp) * kChunk, lane);
            copy_commit();
        };
#pragma unroll 1
        for (int u = 0; u < kSlots; ++u)
            fetch(u, u);
#pragma unroll
        for (int k = 0; k < kQ; ++k) {
            const int i = tid + k * kWarps * 32;
            if (i < ROWS * (DP / 8))
                *reinterpret_cast<uint4 *>(s_q + tile_off<DP>(i / (DP / 8), i % (DP / 8))) = qv[k];
        }
        __syncthreads();
        const unsigned sq = smem_addr(s_q);
        unsigned qf[NT <= 2 ? NT : 1][DP / 16][2];
#pragma unroll
        for (int n = 0; n < (NT <= 2 ? NT : 0); ++n)
#pragma unroll
            for (int k = 0; k < DP / 16; k += 2) {
                unsigned f[4];
                query_pair<DP>(f, sq, n, k, lane);
                qf[n][k][0] = f[0], qf[n][k][1] = f[1], qf[n][k + 1][0] = f[2], qf[n][k + 1][1] = f[3];
            }

        // last position that each of this lane's query rows sees
        int limit[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                limit[n][e] = pos + p.by_g(r0 + 8 * n + 2 * (lane & 3) + e);

        float o[NT][DP / 16][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < DP / 16; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[n][j][e] = 0.f;
            m[n][0] = m[n][1] = -CUDART_INF_F;
            l[n][0] = l[n][1] = 0.f;
        }

        int slot = 0;
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            copy_wait<kSlots - 1>();
            __syncwarp();
            const unsigned keys = ring + slot * Shape::kUnit;
            const int base = src.x0 + (i * kWarps + warp) * kChunk;
            float x[NT][4];
            chunk_scores<T, DP, NT>(x, p, qf, sq, keys, lane, base, src.x1, limit, causal || base + kChunk > src.x1, causal);
            bool partial = false;                    // a key that some query rows, or all, do not see
            if (causal) {
                bool some = false;
                if (lane < kChunk && base + lane >= p.P && base + lane < src.x1) {
                    int age;
                    asm volatile("ld.shared.s32 %0, [%1];" : "=r"(age) : "r"(keys + kChunk * DP * 2 + lane * 4) : "memory");
                    some = age > pos;
                }
                partial = __any_sync(0xffffffffu, some);
            }
            __syncwarp();                            // the keys (and ages) have been read
            fetch(2 * i + kSlots, slot);
            slot = slot + 1 == kSlots ? 0 : slot + 1;
            if (keep && base - src.x0 >= kept0) {
                float *to = s_score + base - src.x0 - kept0 + (lane >> 2);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int r = 8 * n + 2 * (lane & 3) + (e & 1);
                        if (r < nr)
                            to[r * p.score_cap + 8 * (e >> 1)] = x[n][e];
                    }
            }
            // the reference moves only when some score exceeds it by more than the lag (the first keys,
            // rarely later)
            bool grow = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    grow = grow || fmaxf(x[n][e], x[n][2 + e]) > m[n][e] + Ref::kLag;
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(x[n][e], x[n][2 + e]);
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                        const float mn = fmaxf(m[n][e], top - Ref::kBelow);
                        const float f = mn == -CUDART_INF_F ? 1.f : exp2_fast(m[n][e] - mn);
                        m[n][e] = mn;
                        l[n][e] *= f;
#pragma unroll
                        for (int j = 0; j < DP / 16; ++j) {
                            o[n][j][e] *= f;
                            o[n][j][2 + e] *= f;
                        }
                    }
            }
            // the probabilities enter the second product in the values' type: rounded to nearest, like
            // the values themselves; the sum l keeps the unrounded ones
            unsigned pf[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float ref = m[n][e & 1] == -CUDART_INF_F ? 0.f : m[n][e & 1];
                    x[n][e] = exp2_fast(x[n][e] - ref);
                    l[n][e & 1] += x[n][e];
                }
                pf[n][0] = transpose8(Half2<T>::pack(x[n][0], x[n][1]));
                pf[n][1] = transpose8(Half2<T>::pack(x[n][2], x[n][3]));
            }
            copy_wait<kSlots - 1>();
            __syncwarp();
            const unsigned values = ring + slot * Shape::kUnit;
            if (partial)
                add_nonfinite_values<T, DP, NT>(o, x, ring_ptr + slot * Shape::kUnit, lane);
#pragma unroll
            for (int j = 0; j < DP / 16; ++j) {
                unsigned a[4];
                ldsm4_trans(a, values + tile_off<DP>((lane & 7) + ((lane >> 4) << 3), 2 * j + ((lane >> 3) & 1)));
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    mma16816<T>(o[n][j], a, pf[n][0], pf[n][1]);
            }
            __syncwarp();
            fetch(2 * i + 1 + kSlots, slot);
            slot = slot + 1 == kSlots ? 0 : slot + 1;
        }
        copy_wait<0>();

        // the warps' partial results meet in shared memory (the ring is free by now)
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * n + 2 * (lane & 3) + e;
                float sum = l[n][e];
                sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                if (lane < 4) {
                    // a token past n_query counts as one that sees nothing
                    const bool real = r < nr && p.by_g(r0 + r) < nq;
                    s_m[warp * ROWS + r] = real ? m[n][e] : -CUDART_INF_F;
                    s_l[warp * ROWS + r] = real ? sum : 0.f;
                }
                if (r < nr) {
                    float *to = s_o + (warp * ROWS + r) * Shape::kPitch + (lane >> 2);
#pragma unroll
                    for (int j = 0; j < DP / 16; ++j) {
                        to[16 * j] = o[n][j][e];
                        to[16 * j + 8] = o[n][j][2 + e];
                    }
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
                // -1: the warp saw no key of this row; whatever its sums hold does not count.  (Scores that
                // are all NaN leave no maximum either, but a sum of NaN.)
                const bool none = s_m[w * ROWS + r] == -CUDART_INF_F && s_l[w * ROWS + r] == 0.f;
                const float f = exp2_fast(s_m[w * ROWS + r] - ref);
                sum += f * s_l[w * ROWS + r];
                s_m[w * ROWS + r] = none ? -1.f : f;
            }
            s_cm[r] = top;
            s_cl[r] = sum;
        }
        __syncthreads();
        auto axpy = [](float4 &v, float f, const float4 &u) {
            v.x += f * u.x;
            v.y += f * u.y;
            v.z += f * u.z;
            v.w += f * u.w;
        };
        for (int i = tid; i < nr * (DP / 4); i += kWarps * 32) {
            const int r = i / (DP / 4), d = 4 * (i % (DP / 4));
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = s_m[w * ROWS + r];
                const float4 u = *reinterpret_cast<const float4 *>(s_o + (w * ROWS + r) * Shape::kPitch + d);
                if (!(f < 0.f))
                    axpy(v, f, u);
            }
            *reinterpret_cast<float4 *>(s_o + r * Shape::kPitch + d) = v;
        }
        if (p.split > 1)
            cluster.sync();
        else
            __syncthreads();
        if (p.part_ml) {
            cstr_wait_for_earlier_kernels();       // the prefix kernel has finished
            cstr_let_next_kernel_start();
        }

        // ... and the cluster's, through distributed shared memory; each CTA finishes a share
        // of the outputs and the weights of its own slots
        // eight lanes per query row, over its parts (there are about eight at most, unless few rows share
        // a long prompt: then lane i takes parts i, i + 8, ...)
        for (int r = tid >> 3; r < (nr + 3 & ~3); r += kWarps * 4) {   // (whole warps: shuffles below)
            const bool on = r < nr;
            const int sub = tid & 7, t = p.by_g(r0 + (on ? r : 0)), g = (r0 + r) - t * p.G;
            const PartList parts = p.part_ml && on && t < nq ? parts_of(p, kh, b * R + r0 + r) : PartList{0, 0, 0};
            const float2 *ml = p.part_ml + (long long)parts.first * 128 + parts.row;
            float2 first = make_float2(-CUDART_INF_F, 0.f);
            if (sub < parts.n)
                first = ml[(long long)sub * 256];
            float cm = -CUDART_INF_F, cl = 0.f;
            if (on && sub < p.split) {
                cm = p.split > 1 ? *cluster.map_shared_rank(s_cm + r, sub) : s_cm[r];
                cl = p.split > 1 ? *cluster.map_shared_rank(s_cl + r, sub) : s_cl[r];
            }
            float top = fmaxf(first.x, cm);
#pragma unroll 4
            for (int i = sub + 8; i < parts.n; i += 8)
                top = fmaxf(top, ml[(long long)i * 256].x);
#pragma unroll
            for (int off = 4; off > 0; off >>= 1)
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float ref = top == -CUDART_INF_F ? 0.f : top;
            float sum = exp2_fast(cm - ref) * cl + exp2_fast(first.x - ref) * first.y;
#pragma unroll 4
            for (int i = sub + 8; i < parts.n; i += 8) {
                const float2 x = ml[(long long)i * 256];
                sum += exp2_fast(x.x - ref) * x.y;
            }
#pragma unroll
            for (int off = 4; off > 0; off >>= 1)
                sum += __shfl_xor_sync(0xffffffffu, sum, off);
            // nothing seen: +infinity, so that 2^(x - lse) is 0 for every key; NaN makes all outputs NaN
            const float lse = sum == 0.f ? CUDART_INF_F : ref + log2f(sum);
            for (int i = sub; i < parts.n; i += 8) {
                const float pm = i < 8 ? first.x : ml[(long long)i * 256].x;
                // -1: a part that saw no key; it has no outputs
                s_fac[r * p.max_parts + i] = pm == -CUDART_INF_F && lse == lse ? -1.f : exp2_fast(pm - lse);
            }
            if (on && sub == 0) {
                s_lse[r] = lse;
                s_parts[r] = parts;
                if (part == 0 && p.lse_out)
                    p.lse_out[((long long)b * p.T + t) * p.Hq + kh * p.G + g] =
                        sum == 0.f ? -CUDART_INF_F : lse * kLn2;
            }
        }
        __syncthreads();
        // A group of `team` lanes per 4 outputs, each lane over every team-th part: as many lanes as
        // there are for few rows, so that the parts are fetched side by side.  Rows run fastest: the
        // parts keep neighbouring rows together.
        const int pieces = nr * (p.D / 4);
        int team = 1;
        while (team < 32 && 2 * team * pieces <= p.split * kWarps * 32 && team < p.max_parts)
            team *= 2;
        const int sub = tid & (team - 1), at_once = kWarps * 32 / team;
        // two pieces at a time with four parts of each in flight, or the last one with eight (a lane
        // without a piece works on the last one, for the warp's sums)
        for (int i0 = part * at_once; i0 < pieces; i0 += 2 * p.split * at_once) {
            const bool two = i0 + p.split * at_once < pieces;
            const int skip = two ? 0 : 4 * team, step = two ? 4 * team : 8 * team;
            int r[2], d4[2], n = 0;
            const float4 *po[2];
            float4 v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = min(i0 + (two ? h * p.split * at_once : 0) + tid / team, pieces - 1);
                d4[h] = i / nr;
                r[h] = i - d4[h] * nr;
                const PartList parts = s_parts[r[h]];
                po[h] = p.part_o + ((long long)parts.first * (DP / 4) + d4[h]) * 128 + parts.row;
                v[h] = make_float4(0.f, 0.f, 0.f, 0.f);
                n = max(n, parts.n);
            }
#pragma unroll 1
            for (int k0 = sub; k0 < n; k0 += step) {
                float4 u[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k0 + h * skip + k * team < s_parts[r[h]].n)
                            u[h][k] = po[h][(long long)(k0 + h * skip + k * team) * (DP / 4) * 256];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k0 + h * skip + k * team < s_parts[r[h]].n) {
                            const float f = s_fac[r[h] * p.max_parts + k0 + h * skip + k * team];
                            if (!(f < 0.f))
                                axpy(v[h], f, u[h][k]);
                        }
            }
            if (!two)
                axpy(v[0], 1.f, v[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h == 1 && !two)
                    break;
                for (int c = sub; c < p.split; c += team) {
                    const float *so = p.split > 1 ? cluster.map_shared_rank(s_o, c) : s_o;
                    const float cm = p.split > 1 ? *cluster.map_shared_rank(s_cm + r[h], c) : s_cm[r[h]];
                    if (cm != -CUDART_INF_F || s_lse[r[h]] != s_lse[r[h]])
                        axpy(v[h], exp2_fast(cm - s_lse[r[h]]),
                             *reinterpret_cast<const float4 *>(so + r[h] * Shape::kPitch + 4 * d4[h]));
                }
                for (int off = 1; off < team; off <<= 1) {
                    v[h].x += __shfl_xor_sync(0xffffffffu, v[h].x, off);
                    v[h].y += __shfl_xor_sync(0xffffffffu, v[h].y, off);
                    v[h].z += __shfl_xor_sync(0xffffffffu, v[h].z, off);
                    v[h].w += __shfl_xor_sync(0xffffffffu, v[h].w, off);
                }
                if (sub != 0 || i0 + h * p.split * at_once + tid / team >= pieces)
                    continue;
                const int t = p.by_g(r0 + r[h]), g = (r0 + r[h]) - t * p.G;
                char *dst = (char *)p.out + ((long long)b * p.o_sb + (long long)t * p.o_st +
                                             (long long)(kh * p.G + g) * p.o_sh + 4 * d4[h]) * 2;
                *reinterpret_cast<uint2 *>(dst) = make_uint2(Half2<T>::pack(v[h].x, v[h].y), Half2<T>::pack(v[h].z, v[h].w));
            }
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
                const float *score = s_score + (s0 - src.x0 - kept0);
                const int real = min(nr, nq * p.G - r0);           // rows of tokens below n_query
                for (int j0 = tid; j0 < s1 - s0; j0 += 4 * kWarps * 32) {      // four slots at a time
                    float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
                    for (int r = 0; r < real; ++r) {
                        const float lse = s_lse[r];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (j0 + u * kWarps * 32 < s1 - s0)
                                w[u] += exp2_fast(score[r * p.score_cap + j0 + u * kWarps * 32] - lse);
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const long long at = s0 - p.P + j0 + u * kWarps * 32;
                        if (j0 + u * kWarps * 32 < s1 - s0 && real > 0 && CSTR_INB(p.oob, at, p.cap, CSTR_SITE_CACHE))
                            add_once(wrow + at, w[u]);
                    }
                }
            } else {                                // scores once more from the keys
                float lse[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = 8 * n + 2 * (lane & 3) + e;
                        lse[n][e] = r < nr && p.by_g(r0 + r) < nq ? s_lse[r] : CUDART_INF_F;
                    }
                for (int c = kept0 / kChunk + warp; c < n_chunks; c += kWarps) {
                    const int base = src.x0 + c * kChunk;
                    src.fetch(ring, false, base, lane);
                    copy_commit();
                    copy_wait<0>();
                    __syncwarp();
                    float x[NT][4], w[2] = {0.f, 0.f};
                    chunk_scores<T, DP, NT>(x, p, qf, sq, ring, lane, base, src.x1, limit, true, causal);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            // (a select: what a row past n_query scores, its queries being anything, may be NaN)
                            w[e >> 1] += lse[n][e & 1] == CUDART_INF_F ? 0.f : exp2_fast(x[n][e] - lse[n][e & 1]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        w[h] += __shfl_xor_sync(0xffffffffu, w[h], 1);
                        w[h] += __shfl_xor_sync(0xffffffffu, w[h], 2);
                        const int at = base + 8 * h + (lane >> 2);
                        if ((lane & 3) == 0 && at >= s0 && at < s1 && CSTR_INB(p.oob, at - p.P, p.cap, CSTR_SITE_CACHE))
                            add_once(wrow + at - p.P, w[h]);
                    }
                    __syncwarp();
                }
            }
        }
        __syncthreads();
    }
}

template <typename T, int DP, int NT>
int launch(const cstr_cache &c, RowParams p, cudaStream_t stream)
{
    using Shape = RowShape<DP, NT>;
    constexpr int ROWS = 8 * NT;
    constexpr int out = kWarps * ROWS * Shape::kPitch * 4;
    const int fixed = ROWS * DP * 2 + (2 * kWarps + 3) * ROWS * 4 + (Shape::kRing > out ? Shape::kRing : out);
    const int rows = p.G * p.T < ROWS ? p.G * p.T : ROWS;
    int smem = fixed + rows * p.max_parts * 4;
    p.score_cap = 0;
    // the scores stay in shared memory for the weights, if they fit (512 rows 380 us, 505 us where they are
    // computed from the keys again; 64 rows 33.5 / 36.9 us)
    if (p.accumulate) {
        // own slots, at most: a CTA's share of the list may be slots alone.  Whole chunks; behind
        // prefix keys the slots may begin within a chunk.
        const long long share = ((long long)p.P + p.cap + p.split - 1) / p.split + (p.split > 1 ? kChunk : 0);
        const long long own = (share < p.cap ? share : p.cap) + (p.P > 0 ? kChunk : 0);
        const long long want = (own + kChunk - 1) / kChunk * kChunk;
        if (smem + want * rows * 4 <= kMostSmem) {
            p.score_cap = (int)want;
            smem += (int)(want * rows * 4);
        }
    }
    auto kernel = row_attention_kernel<T, DP, NT>;
    static std::atomic<bool> allowed[64];
    const int rc = cstr_allow_smem(kernel, allowed, c.device, kMostSmem);
    if (rc)
        return rc;
    return cstr_launch(kernel, (long long)p.B * p.Hk * p.split, kWarps * 32, p.split, smem, stream, p);
}

template <typename T>
int launch_typed(const cstr_cache &c, const RowParams &p, cudaStream_t stream)
{
    const bool wide = c.head_dim > 64;
    const int rows = p.G * p.T;
    // as few passes over the keys as there are blocks of 32 query rows, and no wider than needed: the
    // widest for all costs registers and shared memory (64 rows of 4 query rows 47.0 us, 33.5 us so;
    // 512 rows 558 / 380 us; 64 rows of 20 query rows 96.9 / 88.9 us)
    if (rows <= 8)
        return wide ? launch<T, 128, 1>(c, p, stream) : launch<T, 64, 1>(c, p, stream);
    if (rows <= 16)
        return wide ? launch<T, 128, 2>(c, p, stream) : launch<T, 64, 2>(c, p, stream);
    if (rows <= 24)
        return wide ? launch<T, 128, 3>(c, p, stream) : launch<T, 64, 3>(c, p, stream);
    return wide ? launch<T, 128, 4>(c, p, stream) : launch<T, 64, 4>(c, p, stream);
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
    p.by_g.set(p.G);
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
        p.narrow = (long long)c.n_kv_heads * s.pairs * s.tiles * s.grid < 0x7fffffffLL;
        p.max_parts = s.grid / (c.n_kv_heads * s.pairs) + 2;
    }
    p.scale_log2 = a.scale_log2;
    p.accumulate = a.accumulate;
    p.oob = CSTR_OOB_RECORD();
    // share a row's keys among CTAs while all of them still run at once (four per SM) and each has
    // 64 keys (6 rows x 4 heads of 512 slots behind 65,000 tokens: 39.2 us, unshared 48.8 us, by four
    // at most 41.3 us; the batches of 64 and 512 rows are not shared)
    const long long items = (long long)p.B * p.Hk;
    p.split = 1;
    while (p.split < 8 && items * p.split * 2 <= 4LL * c.sm_count &&
           (long long)p.P + p.cap >= 2LL * p.split * 64)
        p.split *= 2;
    if (items * p.split > 0x7fffffffLL)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_cache_attention: batch x heads too large for one launch");
    return c.dtype == CSTR_BF16 ? launch_typed<__nv_bfloat16>(c, p, stream)
                                : launch_typed<__half>(c, p, stream);
}
