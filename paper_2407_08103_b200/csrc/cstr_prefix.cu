// Attention of a whole batch over the prompt that its rows share, on the tensor
// cores: for one key / value head all query rows of the batch form one matrix of
// M = batch x tokens x group rows, so the prompt's keys and values are read once
// per 256 of them instead of once per row.
//
// Mathematics: as in the row kernel, one pass over the keys with the running
// maximum m and sum l of a base-2 softmax and o = sum 2^(x - m) v, over a part
// of the prompt; parts (m, l, o) are joined by the row kernel.
//
// One CTA works on two "streams", each with its own 128-row scores S and output
// O in tensor memory (4 x 128 columns = all 512):
//   more than 128 query rows left: two tiles of query rows over the same keys;
//   else: one tile, the streams taking alternate key tiles.
// While the 128 threads of one stream turn its S into probabilities P, the
// tensor cores work for the other stream.  One thread issues all products,
// S = Q K^T (both operands from shared memory) and O += P V (P from tensor
// memory, over its own S), one thread issues the copies into a ring of tiles, and
// two warps bring the next row group's queries while the last one is finished.
//
// Split: the units (key tile x group of 256 query rows) are dealt out evenly and
// contiguously, to one CTA per SM where there are enough, so a CTA starts or ends
// within a row group and no SM idles in a last wave; each (CTA, row group) segment
// leaves one part.
//
// Bound: at 512 rows x 4 heads a key / value head, 8 of these, 16,384 tokens, head_dim
// 128, bf16 (137 GFLOP) it takes 139 us, 990 TFLOP/s; the tensor cores wait for the
// chain scores -> probabilities -> second product of the two streams, about 3,300
// cycles per 128 keys x 256 rows.  It is not the exponentials alone: taking 2 to 4
// of 8 pairs of them on the multiply-add units instead was slower (+3 to +21 us).
// With few rows it is bound by the bytes of the prompt (6 rows x 16 heads, 65,000
// tokens: 39 us with the join, 133 MB, 3.5 TB/s) and by the fixed cost of the
// set-up, the parts and their join.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <math.h>
#include <string.h>

#include "cstr_cache.cuh"

namespace {

constexpr int kThreads = 384;        // warps 0-3: copies, products, query tiles (two); 4-7, 8-11: streams
constexpr int kTile = 128;           // query rows and keys of a tile
constexpr int kWaitLimit = 1 << 22;

template <int DP> struct Shape {
    static constexpr int kTileBytes = kTile * DP * 2;
    static constexpr int kSlots = DP == 128 ? 5 : 8;
    static constexpr int kSmem = (2 + kSlots) * kTileBytes + 1024 /* alignment */ + 256;
};

struct PrefixParams {
    const void *q;
    int q_sb, q_st, q_sh;            // bytes / 16
    float *part_o;
    float2 *part_ml;
    int *status;
    int M, T, G, R, D, P, Hk;        // R = T G query rows of one batch row
    int tiles, pairs, grid;
    float scale_log2;                // > 0: for a negative scale the first product negates the queries
    unsigned negate;                 // bit of the instruction descriptor
    cstr_divisor by_r, by_g;
    int wait_limit;                  // kWaitLimit but in tests
};

#ifdef CSTR_TESTING
int g_test_wait_limit = kWaitLimit;
#endif

__device__ __forceinline__ unsigned smem_addr(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// two fp32 operations per instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n.reg .b64 x, y, z, w;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 z, {%6, %7};\n"
        "fma.rn.f32x2 w, x, y, z;\nmov.b64 {%0, %1}, w;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n.reg .b64 x, y, w;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\n"
        "add.rn.f32x2 w, x, y;\nmov.b64 {%0, %1}, w;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

template <typename T> __device__ __forceinline__ unsigned pack2(float lo, float hi);
template <> __device__ __forceinline__ unsigned pack2<__nv_bfloat16>(float lo, float hi)
{
    unsigned u;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
    return u;
}
template <> __device__ __forceinline__ unsigned pack2<__half>(float lo, float hi)
{
    unsigned u;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
    return u;
}

// ---- barriers: every wait ends, after abort[1] tries with the CTA's abort flag, abort[0], set ----

__device__ __forceinline__ void bar_init(unsigned bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(unsigned bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(unsigned bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(unsigned bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __noinline__ bool bar_wait_slow(unsigned bar, unsigned parity, volatile int *abort)
{
    const int limit = abort[1];
    for (int i = 0; i < limit; ++i) {
        if (bar_try(bar, parity))
            return true;
        if (abort[0])
            return false;
    }
    abort[0] = 1;
    return false;
}
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity, volatile int *abort)
{
#ifdef CSTR_TESTING
    if (abort[1] == 0) {                         // one look, without the pause of a try
        unsigned ok;
        asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}\n"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        return ok || bar_wait_slow(bar, parity, abort);
    }
#endif
    return bar_try(bar, parity) || bar_wait_slow(bar, parity, abort);
}

// ---- tensor memory and products ---------------------------------------------

__device__ __forceinline__ void tmem_ld32(float (&r)[32], unsigned addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
          "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
          "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
          "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_st32(unsigned addr, const float (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::"f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]),
          "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]), "f"(r[14]), "f"(r[15]),
          "f"(r[16]), "f"(r[17]), "f"(r[18]), "f"(r[19]), "f"(r[20]), "f"(r[21]), "f"(r[22]), "f"(r[23]),
          "f"(r[24]), "f"(r[25]), "f"(r[26]), "f"(r[27]), "f"(r[28]), "f"(r[29]), "f"(r[30]), "f"(r[31]),
          "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(unsigned addr, const unsigned (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(addr)
        : "memory");
}
// Loads complete.  The registers are operands, so that no use of them moves before the wait.
__device__ __forceinline__ void tmem_wait_ld(float (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]),
                   "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]),
                   "+f"(r[16]), "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]),
                   "+f"(r[24]), "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])
                 :: "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 1 in one lane of the warp, the same one every time
__device__ __forceinline__ unsigned elected()
{
    unsigned leader;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(leader));
    return leader;
}

// The products are issued by one lane (`leader`) of a warp that runs through the loop as a whole:
// every operand is then the same in all lanes and stays in the uniform registers that the
// instructions take them from, instead of being moved there one by one.
__device__ __forceinline__ void commit(unsigned leader, unsigned bar)
{
    asm volatile("{\n.reg .pred l;\nsetp.ne.u32 l, %0, 0;\n"
                 "@l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n}\n"
                 ::"r"(leader), "r"(bar) : "memory");
}

// Shared-memory operand with 128-byte rows in the 128-byte swizzle.  Low word: address and, for a
// transposed operand, the bytes (kLead) between blocks of 64 elements along its row dimension;
// high word: 1,024 bytes between groups of eight rows, version, swizzle.
constexpr unsigned kOperandHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
constexpr unsigned kLead = kTile * 128;
__device__ __forceinline__ unsigned operand(unsigned addr, unsigned lead)
{
    return ((addr & 0x3ffffu) >> 4) | ((lead >> 4) << 16);
}

__device__ __forceinline__ void mma_ss(unsigned leader, unsigned d, unsigned a, unsigned b, unsigned idesc, unsigned add)
{
    asm volatile("{\n.reg .pred l, p;\n.reg .b64 x, y;\nsetp.ne.u32 l, %0, 0;\nsetp.ne.u32 p, %5, 0;\n"
                 "mov.b64 x, {%2, %6};\nmov.b64 y, {%3, %6};\n"
                 "@l tcgen05.mma.cta_group::1.kind::f16 [%1], x, y, %4, p;\n}\n"
                 ::"r"(leader), "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(add), "n"(kOperandHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(unsigned leader, unsigned d, unsigned a, unsigned b, unsigned idesc, unsigned add)
{
    asm volatile("{\n.reg .pred l, p;\n.reg .b64 y;\nsetp.ne.u32 l, %0, 0;\nsetp.ne.u32 p, %5, 0;\n"
                 "mov.b64 y, {%3, %6};\n"
                 "@l tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], y, %4, p;\n}\n"
                 ::"r"(leader), "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(add), "n"(kOperandHigh) : "memory");
}

__device__ __forceinline__ void tma_tile(unsigned dst, const CUtensorMap *map, int x, int key, int head, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"((unsigned long long)map), "r"(x), "r"(key), "r"(head), "r"(bar) : "memory");
}

// The part of one CTA's unit range that lies in one row group.
struct Segment {
    int item, tile0, tiles, rows;    // key tiles [tile0, tile0 + tiles); query rows of the group
    bool pair_rows;                  // two row tiles (else: one, key tiles alternating)
};

struct Walk {
    const PrefixParams &p;
    long long at, end;
    __device__ __forceinline__ explicit Walk(const PrefixParams &p_) : p(p_)
    {
        const long long units = (long long)p.Hk * p.pairs * p.tiles;
        at = units * blockIdx.x / p.grid;
        end = units * (blockIdx.x + 1) / p.grid;
    }
    __device__ __forceinline__ bool next(Segment &s)
    {
        if (at >= end)
            return false;
        s.item = end < (1ll << 31) ? (int)((unsigned)at / (unsigned)p.tiles) : (int)(at / p.tiles);
        s.tile0 = (int)(at - (long long)s.item * p.tiles);
        s.tiles = (int)min((long long)(p.tiles - s.tile0), end - at);
        const int pair = s.item % p.pairs;
        s.rows = min(p.M - pair * 2 * kTile, 2 * kTile);
        s.pair_rows = s.rows > kTile;
        at += s.tiles;
        return true;
    }
};

// Place of a tile in a segment's sequence of copies: the first `lead` key tiles, then value tile i
// and key tile i + lead in turn - the order in which the products use them.
__device__ __forceinline__ int place_k(int i, int lead) { return i < lead ? i : 2 * i - lead + 1; }
__device__ __forceinline__ int place_v(int i, int lead, int n)
{
    return i <= n - lead ? lead + 2 * i : n + i;
}

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 1)
prefix_attention_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                        const __grid_constant__ PrefixParams p)
{
    using S = Shape<DP>;
    using Ref = cstr_softmax_reference<T>;       // (moving it costs a round trip of O through registers)
    constexpr int kSlots = S::kSlots;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) unsigned long long s_bar[2 * kSlots + 12];
    __shared__ float2 s_ml[kTile];               // second stream's maximum and sum, one-tile segments
    __shared__ unsigned s_tmem;
    __shared__ int s_abort[2];                   // a wait has run out; tries of a wait
    __shared__ unsigned s_copies;                // tiles that were sent for (in shared memory, not in everyone's registers)
    const unsigned raw = smem_addr(smem_raw);
    const unsigned q_tile = (raw + 1023u) & ~1023u;              // [2][kTile][DP], swizzled
    const unsigned ring = q_tile + 2 * S::kTileBytes;
    const unsigned bars = smem_addr(s_bar);
    auto full = [&](int slot) { return bars + 8u * slot; };
    auto empty = [&](int slot) { return bars + 8u * (kSlots + slot); };
    const unsigned q_full = bars + 8u * (2 * kSlots), drain = q_full + 56, q_free = q_full + 64, ml_full = q_full + 72, ml_free = q_full + 80,
                   q_first = q_full + 88;
    auto s_full = [&](int s) { return q_full + 8u * (1 + s); };
    auto p_full = [&](int s) { return q_full + 8u * (3 + s); };
    auto o_full = [&](int s) { return q_full + 8u * (5 + s); };

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int *abort = s_abort;
    if (tid == 0) {
        s_abort[0] = 0;
        s_abort[1] = p.wait_limit;
        for (int i = 0; i < kSlots; ++i) {
            bar_init(full(i), 1);
            bar_init(empty(i), 1);
        }
        bar_init(q_full, 64);
        bar_init(q_first, 320);
        for (int s = 0; s < 2; ++s) {
            bar_init(s_full(s), 1);
            bar_init(p_full(s), 4);
            bar_init(o_full(s), 1);
        }
        bar_init(drain, 1);
        bar_init(q_free, 1);
        bar_init(ml_full, 4);
        bar_init(ml_free, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    __syncthreads();
    fence_after();
    // Up to here nothing that an earlier kernel may still write has been read.  The row kernel may start
    // from here on; it waits for this one's parts.
    cstr_wait_for_earlier_kernels();
    cstr_let_next_kernel_start();
    const unsigned tmem = s_tmem;
    const unsigned t_s = tmem, t_o = tmem + 2 * kTile;           // S (and P over it), O: + stream * 128

    // a segment's query rows into the swizzled tiles; thread `index` of `threads`
    auto load_queries = [&](const Segment &g, int index, int threads) {
        const int head = g.item / p.pairs, row0 = (g.item % p.pairs) * 2 * kTile;
        const int q_rows = g.pair_rows ? 2 * kTile : kTile;
        const int ch = index % (DP / 8);
#pragma unroll 4
        for (int r = index / (DP / 8); r < q_rows; r += threads / (DP / 8)) {
            const bool ok = r < g.rows && ch * 8 < p.D;          // else zeroes
            const int m = ok ? row0 + r : 0, b = p.by_r(m), in = m - b * p.R, t = p.by_g(in), gh = in - t * p.G;
            const uint4 *from = reinterpret_cast<const uint4 *>(p.q) + ((long long)b * p.q_sb + (long long)t * p.q_st +
                                (long long)(head * p.G + gh) * p.q_sh + (ok ? ch : 0));
            const unsigned to = q_tile + (r / kTile) * S::kTileBytes + (ch / 8) * (kTile * 128) + (r % kTile) * 128 +
                                (((ch ^ r) & 7) << 4);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(ok ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    };

    Walk walk(p);
    Segment g;
    if (warp == 0) {
        if (lane == 0) {                                         // copies
            unsigned copies = 0;
            bool alive = true;
            auto put = [&](const CUtensorMap *map, int key_tile, int head) {
                const int slot = copies % kSlots;
                alive = alive && bar_wait(empty(slot), ((copies / kSlots) & 1u) ^ 1u, abort);
                if (!alive)
                    return;
                bar_expect(full(slot), S::kTileBytes);
#pragma unroll
                for (int x = 0; x < DP / 64; ++x)
                    tma_tile(ring + slot * S::kTileBytes + x * (kTile * 128), map, x * 64, key_tile * kTile, head, full(slot));
                ++copies;
            };
            while (alive && walk.next(g)) {
                const int head = g.item / p.pairs;
                const int lead = min(g.pair_rows ? 1 : 2, g.tiles);
                for (int i = 0; i < lead; ++i)
                    put(&map_k, g.tile0 + i, head);
                for (int i = 0; i < g.tiles && alive; ++i) {
                    put(&map_v, g.tile0 + i, head);
                    if (i + lead < g.tiles)
                        put(&map_k, g.tile0 + i + lead, head);
                }
            }
            s_copies = copies;
        }
        __syncwarp();
    } else if (warp == 1) {
        // products
        constexpr unsigned type = __is_same(T, __nv_bfloat16) ? 1u : 0u;
        constexpr unsigned idesc = (1u << 4) | (type << 7) | (type << 10) | ((kTile / 16) << 24);
        const unsigned idesc_s = idesc | ((kTile / 8) << 17) | p.negate;
        constexpr unsigned idesc_o = idesc | (1u << 16) | ((DP / 8) << 17);
        const unsigned leader = elected();
        unsigned base = 0, seg = 0, p_count[2] = {0, 0};
        bool alive = true;
        auto wait = [&](unsigned bar, unsigned parity) {
            alive = alive && __all_sync(0xffffffffu, bar_wait(bar, parity, abort));
        };
        while (alive && walk.next(g)) {
            const int lead = min(g.pair_rows ? 1 : 2, g.tiles);
            const int visits = g.pair_rows ? 2 * g.tiles : g.tiles;
            const int shift = g.pair_rows ? 1 : 0;
            if (seg == 0)
                wait(q_first, 0);
            else
                wait(q_full, (seg - 1) & 1u);
            ++seg;
            auto scores = [&](int n) {
                const unsigned at = base + place_k(n >> shift, lead);
                const int slot = at % kSlots;
                wait(full(slot), (at / kSlots) & 1u);
                if (!alive)
                    return;
                fence_after();
                const int s = n & 1;
                const unsigned qa = operand(q_tile + (g.pair_rows ? s : 0) * S::kTileBytes, 16);
                const unsigned ka = operand(ring + slot * S::kTileBytes, 16);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const unsigned off = ((k / 4) * (kTile * 128) + (k % 4) * 32) >> 4;
                    mma_ss(leader, t_s + s * kTile, qa + off, ka + off, idesc_s, k > 0);
                }
                commit(leader, s_full(s));
                if (!g.pair_rows || s == 1)
                    commit(leader, empty(slot));
                if (n == visits - 1)
                    commit(leader, q_free);
            };
            scores(0);
            if (visits > 1)
                scores(1);
            for (int n = 0; n < visits; ++n) {
                const int s = n & 1;
                const unsigned at = base + place_v(n >> shift, lead, g.tiles);
                const int slot = at % kSlots;
                wait(full(slot), (at / kSlots) & 1u);
                wait(p_full(s), p_count[s] & 1u);
                if (!alive)
                    break;
                ++p_count[s];
                fence_after();
                const unsigned va = operand(ring + slot * S::kTileBytes, kLead);
#pragma unroll
                for (int k = 0; k < kTile / 16; ++k)
                    mma_ts(leader, t_o + s * kTile, t_s + s * kTile + 8 * k, va + k * (2048 >> 4), idesc_o,
                           k > 0 ? 1u : (unsigned)(n >= 2));
                commit(leader, o_full(s));
                if (!g.pair_rows || s == 1)
                    commit(leader, empty(slot));
                if (n + 2 < visits)
                    scores(n + 2);
            }
            base += 2 * g.tiles;
        }
        __syncwarp();
    } else if (warp < 4) {                                       // query tiles, by two warps
        unsigned seg = 0;
        bool alive = true;
        for (; alive && walk.next(g); ++seg) {
            // the previous segment's last scores have been computed: its tiles may be replaced
            if (seg > 0 && !(alive = __all_sync(0xffffffffu, bar_wait(q_free, (seg - 1) & 1u, abort))))
                break;
            // (the first segment's with the streams' help)
            load_queries(g, tid - 64, seg == 0 ? 320 : 64);
            bar_arrive(seg == 0 ? q_first : q_full);
        }
        __syncwarp();
    } else {
        const int s = (warp - 4) >> 2, row = ((warp & 3) << 5) + lane;    // stream; row of its tile = TMEM lane
        const unsigned lane_base = (unsigned)((warp & 3) << 5) << 16;
        const unsigned my_s = t_s + s * kTile + lane_base, my_o = t_o + s * kTile + lane_base;
        unsigned done = 0, joined = 0;                           // visits of this stream, joins so far
        bool alive = true, started = false;
        while (alive && walk.next(g)) {
            if (!started) {
                load_queries(g, tid - 64, 320);
                bar_arrive(q_first);
                started = true;
            }
            const int my_row = g.pair_rows ? s * kTile + row : row;      // row of the group
            const bool warp_on = my_row - lane < g.rows;
            const int visits = g.pair_rows ? 2 * g.tiles : g.tiles;
            float m = -CUDART_INF_F, l = 0.f;
            int mine = 0;                                        // visits of this stream in this segment
            for (int n = s; n < visits; n += 2, ++mine, ++done) {
                if (!(alive = __all_sync(0xffffffffu, bar_wait(s_full(s), done & 1u, abort))))
                    break;
                fence_after();
                if (warp_on) {
                    const int valid = p.P - (g.tile0 + (g.pair_rows ? n >> 1 : n)) * kTile;
                    if (mine == 0) {                             // the first keys' maximum sets the first reference
                        float top = -CUDART_INF_F;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            float y[32];
                            tmem_ld32(y, my_s + 32 * c);
                            tmem_wait_ld(y);
#pragma unroll
                            for (int i = 0; i < 32; i += 2)
                                top = max3(top, 32 * c + i < valid ? y[i] : -CUDART_INF_F,
                                           32 * c + i + 1 < valid ? y[i + 1] : -CUDART_INF_F);
                        }
                        m = top * p.scale_log2 - Ref::kBelow;
                    }
                    // One pass over the scores with the reference so far; only if some row's maximum
                    // turns out to exceed it by more than the lag (rarely) the reference moves and the
                    // pass is taken again.  P replaces S afterwards.
                    unsigned w[4][16];
                    float sum;
                    for (;;) {
                        const float ref = m == -CUDART_INF_F ? 0.f : m;
                        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), ref2 = make_float2(-ref, -ref);
                        float x[2][32];                          // a quarter is worked on, one on its way
                        float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                        float top[2] = {-CUDART_INF_F, -CUDART_INF_F};
                        tmem_ld32(x[0], my_s);
                        tmem_wait_ld(x[0]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            float (&y)[32] = x[c & 1], (&next)[32] = x[(c + 1) & 1];
                            if (c < 3)
                                tmem_ld32(next, my_s + 32 * (c + 1));
                            if (valid < 32 * c + 32) {           // keys past the prompt's end
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (32 * c + i >= valid)
                                        y[i] = -CUDART_INF_F;
                            }
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                top[(i >> 1) & 1] = max3(top[(i >> 1) & 1], y[i], y[i + 1]);
                                float2 e = fma2(make_float2(y[i], y[i + 1]), scale2, ref2);
                                e.x = exp2_fast(e.x);
                                e.y = exp2_fast(e.y);
                                sum2[(i >> 1) & 1] = add2(sum2[(i >> 1) & 1], e);
                                // rounded to the values' type for the second product; the sum is not
                                w[c][i / 2] = pack2<T>(e.x, e.y);
                            }
                            if (c < 3)
                                tmem_wait_ld(next);
                        }
                        sum = (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
                        const float seen = fmaxf(top[0], top[1]) * p.scale_log2;
                        const bool grow = seen > m + Ref::kLag;
                        if (!__any_sync(0xffffffffu, grow))
                            break;
                        const float to = grow ? seen - Ref::kBelow : m;
                        const float f = m == to ? 1.f : exp2_fast(m - to);
                        l *= f;
                        m = to;
                        if (mine > 0) {                          // O so far counts from the old reference
                            if (!(alive = __all_sync(0xffffffffu, bar_wait(o_full(s), (done - 1) & 1u, abort))))
                                break;
                            fence_after();
#pragma unroll
                            for (int c = 0; c < DP / 32; ++c) {
                                float o[32];
                                tmem_ld32(o, my_o + 32 * c);
                                tmem_wait_ld(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    o[i] *= f;
                                tmem_st32(my_o + 32 * c, o);
                            }
                        }
                    }
                    if (!alive)
                        break;
                    l += sum;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        tmem_st16(my_s + 16 * c, w[c]);
                    tmem_wait_st();
                }
                fence_before();
                __syncwarp();
                if (lane == 0)
                    bar_arrive(p_full(s));
            }
            if (!alive)
                break;
            if (mine > 0) {
                if (!(alive = __all_sync(0xffffffffu, bar_wait(o_full(s), (done - 1) & 1u, abort))))
                    break;
                fence_after();
            }
            // One-tile segments: the first stream takes the second one's O (the same tensor memory
            // lanes) and statistics, and writes one part for both.
            float m1 = -CUDART_INF_F, l1 = 0.f;
            if (!g.pair_rows) {
                if (s == 1) {
                    s_ml[row] = make_float2(m, l);
                    fence_before();
                    __syncwarp();
                    if (lane == 0)
                        bar_arrive(ml_full);
                    alive = __all_sync(0xffffffffu, bar_wait(ml_free, joined & 1u, abort));
                    fence_after();
                } else {
                    if (!(alive = __all_sync(0xffffffffu, bar_wait(ml_full, joined & 1u, abort))))
                        break;
                    fence_after();
                    m1 = s_ml[row].x;
                    l1 = s_ml[row].y;
                }
                ++joined;
            }
            if (s == 0 || g.pair_rows) {
                const float top = fmaxf(m, m1), ref = top == -CUDART_INF_F ? 0.f : top;
                const float f0 = exp2_fast(m - ref), f1 = exp2_fast(m1 - ref);
                const bool both = !g.pair_rows && visits > 1;
                // O as [DP / 4][128][4], so that a warp's rows are adjacent
                const long long block = ((long long)blockIdx.x + g.item) * 2 + s;
                if (warp_on) {
                    float4 *dst = reinterpret_cast<float4 *>(p.part_o) + block * (DP / 4) * kTile + row;
#pragma unroll
                    for (int c = 0; c < DP / 32; ++c) {
                        float o[32];
                        tmem_ld32(o, my_o + 32 * c);
                        tmem_wait_ld(o);
                        if (both) {
                            float o1[32];
                            tmem_ld32(o1, my_o + kTile + 32 * c);
                            tmem_wait_ld(o1);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                o[i] = f0 * o[i] + f1 * o1[i];
                        }
                        if (my_row < g.rows)
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                dst[(c * 8 + i) * kTile] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                    if (my_row < g.rows)
                        p.part_ml[block * kTile + row] = both ? make_float2(top, f0 * l + f1 * l1) : make_float2(m, l);
                }
                if (!g.pair_rows) {
                    fence_before();
                    __syncwarp();
                    if (lane == 0)
                        bar_arrive(ml_free);
                }
            }
            if (!alive)
                break;
            fence_before();
        }
    }
    __syncthreads();
    if (abort[0]) {                              // (nobody sets it any more)
        // No role waits for what it has in flight when another one gives up, so it ends here, before the
        // CTA leaves its shared and tensor memory.
        if (tid == 0) {
            const unsigned copies = s_copies;
            for (unsigned i = copies > kSlots ? copies - kSlots : 0; i < copies; ++i)
                for (int k = 0; k < kWaitLimit && !bar_try(full(i % kSlots), (i / kSlots) & 1u); ++k) {}
            atomicAdd(p.status, 1);
        } else if (warp == 1) {
            commit(elected(), drain);
            for (int k = 0; k < kWaitLimit && !bar_try(drain, 0); ++k) {}
        }
        // its parts become NaN, and with them their rows' outputs: what an earlier call left in their
        // place must not pass for an answer
        Walk again(p);
        while (again.next(g))
            for (int r = tid; r < g.rows; r += kThreads)
                p.part_ml[(((long long)blockIdx.x + g.item) * 2 + r / kTile) * kTile + r % kTile] = make_float2(0.f, CUDART_NAN_F);
        __syncthreads();
    }
    if (warp == 2) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

template <typename T, int DP>
int launch(const cstr_cache &c, const PrefixParams &p, cudaStream_t stream)
{
    auto kernel = prefix_attention_kernel<T, DP>;
    static std::atomic<bool> allowed[64];
    const int rc = cstr_allow_smem(kernel, allowed, c.device, Shape<DP>::kSmem);
    if (rc)
        return rc;
    CUtensorMap k, v;
    memcpy(&k, c.map_k, sizeof k);
    memcpy(&v, c.map_v, sizeof v);
    return cstr_launch(kernel, p.grid, kThreads, 1, Shape<DP>::kSmem, stream, k, v, p);
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

}  // namespace

cstr_prefix_plan cstr_plan_prefix(const cstr_cache &c, int tokens)
{
    cstr_prefix_plan s;
    const long long rows = (long long)c.batch * tokens * (c.n_heads / c.n_kv_heads);
    s.pairs = (int)((rows + 2 * kTile - 1) / (2 * kTile));
    s.tiles = (int)((c.prefix_len + kTile - 1) / kTile);
    const long long units = (long long)c.n_kv_heads * s.pairs * s.tiles;
    // Every CTA leaves a part of up to 128 KB per row group that it works for, as much as two key tiles
    // read, and the row kernel has to join them.  So with two tiles of query rows a CTA gets two units
    // (64 rows x 32 / 8 heads, 4,096 tokens 34.2 us, with one unit 35.7 us; 64 rows x 4 tokens x 8 / 1 heads,
    // 2,048: 26.3 / 38.1; only the shortest prompts lose, 64 rows x 16 / 2 heads, 1,024: 17.4 / 16.3), but there
    // is a CTA per row group at least.  For the same reason no row group gets more than 40 CTAs, though one to
    // three key / value heads leave SMs idle by that: 65,000 tokens, 8 query heads a key / value head, 1 row x
    // 1 head 30.3 us, without the limit 47.2; 1 x 2 32.5 / 39.0; 4 rows x 4 tokens x 1 head 55.2 / 134.9,
    // x 3 heads 66.0 / 79.4; from four heads on it does not act.
    const long long items = (long long)c.n_kv_heads * s.pairs;
    long long grid = rows > kTile ? (units + 1) / 2 : units;
    grid = grid < items ? items : grid;
    grid = grid > 40 * items ? 40 * items : grid;
    s.grid = (int)(grid < c.sm_count ? grid : c.sm_count);
    return s;
}

int cstr_prefix_init(cstr_cache *c)
{
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    CSTR_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found));
    if (!fn || found != cudaDriverEntryPointSuccess)
        return cstr_fail(CSTR_ERR_CUDA, "cstr_cache_create: the driver has no cuTensorMapEncodeTiled");
    for (int i = 0; i < 2; ++i) {
        CUtensorMap map;
        const cuuint64_t dims[3] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->prefix_len, (cuuint64_t)c->n_kv_heads};
        const int64_t st = i ? c->pv_st : c->pk_st, sh = i ? c->pv_sh : c->pk_sh;
        // the stride of a dimension of extent 1 is never used, but has to be a valid one
        const cuuint64_t strides[2] = {(cuuint64_t)(c->prefix_len > 1 ? st * 2 : 16),
                                       (cuuint64_t)(c->n_kv_heads > 1 ? sh * 2 : 16)};
        const cuuint32_t box[3] = {64, kTile, 1}, ones[3] = {1, 1, 1};
        const CUresult r = ((EncodeTiled)fn)(
            &map, c->dtype == CSTR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
            const_cast<void *>(i ? c->prefix_v : c->prefix_k), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r != CUDA_SUCCESS)
            return CSTR_OK;              // strides that the copy engine cannot take: the row kernel reads the prompt
        static_assert(sizeof map == sizeof c->map_k, "tensor map size");
        memcpy(i ? c->map_v : c->map_k, &map, sizeof map);
    }
    // parts: every (CTA, row group) segment has one; CTA index + group index numbers them
    const cstr_prefix_plan s = cstr_plan_prefix(*c, c->max_tokens);
    const size_t blocks = ((size_t)c->sm_count + (size_t)c->n_kv_heads * s.pairs) * 2;
    const size_t dp = c->head_dim > 64 ? 128 : 64;
    CSTR_CUDA_TRY(cudaMalloc((void **)&c->part_o, blocks * kTile * dp * sizeof(float)));
    CSTR_CUDA_TRY(cudaMalloc((void **)&c->part_ml, blocks * kTile * sizeof(float2)));
    c->has_maps = 1;
    return CSTR_OK;
}

int cstr_launch_prefix(const cstr_cache &c, const cstr_row_args &a, cudaStream_t stream)
{
    PrefixParams p;
    memset(&p, 0, sizeof p);
    const cstr_prefix_plan s = cstr_plan_prefix(c, a.tokens);
    p.q = a.q;
    p.q_sb = (int)(a.q_sb / 8), p.q_st = (int)(a.q_st / 8), p.q_sh = (int)(a.q_sh / 8);
    p.part_o = c.part_o;
    p.part_ml = (float2 *)c.part_ml;
    p.status = c.status;
    p.T = a.tokens;
    p.G = c.n_heads / c.n_kv_heads;
    p.R = p.T * p.G;
    p.M = c.batch * p.R;
    p.by_r.set(p.R);
    p.by_g.set(p.G);
    p.D = c.head_dim;
    p.P = (int)c.prefix_len;
    p.Hk = c.n_kv_heads;
    p.tiles = s.tiles;
    p.pairs = s.pairs;
    p.grid = s.grid;
    p.wait_limit = kWaitLimit;
#ifdef CSTR_TESTING
    p.wait_limit = g_test_wait_limit;
#endif
    p.negate = a.scale_log2 < 0.f ? 1u << 13 : 0u;
    // A scale of 0 would turn the -infinity of keys past the prompt's end into NaN.  2^-126 in its place
    // leaves every weight at 1 to 2^-26 for scores below 2^100.
    p.scale_log2 = fmaxf(fabsf(a.scale_log2), 0x1p-126f);
    const bool wide = c.head_dim > 64;
    if (c.dtype == CSTR_BF16)
        return wide ? launch<__nv_bfloat16, 128>(c, p, stream) : launch<__nv_bfloat16, 64>(c, p, stream);
    return wide ? launch<__half, 128>(c, p, stream) : launch<__half, 64>(c, p, stream);
}

#ifdef CSTR_TESTING
extern "C" int cstr_test_set_wait_limit(int32_t tries)
{
    if (tries < -1)
        return cstr_fail(CSTR_ERR_ARG, "cstr_test_set_wait_limit: tries = %d, need -1 or more", tries);
    g_test_wait_limit = tries < 0 ? kWaitLimit : tries;
    return CSTR_OK;
}
#endif
