// Clipped policy loss with a KL term over the constrained distribution, forward
// and gradient, in one kernel.
//
// Mathematics, in base 2 with c = log2(e) / temperature: one pass for the running
// maximum m of the allowed logits x_v and s = sum 2^(c (x_v - m)); log2 p_a =
// c (x_a - m) - log2 s; ratio, loss and d loss / d logp from that; a second pass
// for p_v = 2^(c (x_v - m)) / s.  The maximum is subtracted before the scaling: c m
// rounded would be off by whole powers of two where all allowed logits lie far from
// zero (a model's own mask of -1e9), by 1e-4 at 1e4 already.
//
// Bound: the row is read from memory once and the gradient written once; the
// second pass finds the row in the L2 cache.  For that the rows in flight have to
// fit there: a cluster of up to 16 CTAs shares a row, 64 KB each (512 x 256,000
// fp32: 241 us, 1.05 GB of DRAM traffic, 4.4 TB/s; with 8 CTAs of 128 KB 270 us; 2,048 x
// 32,000 bf16 69 us, 3.9 TB/s, where 22 instructions an element weigh as much).  All 2,048
// threads of an SM are used, at 32 registers, since what is left is the latency
// of the passes and of the join between them.  Measured and dropped: the row held
// in registers between the passes (344 us), and persistent CTAs with a ring of
// bulk copies in shared memory (302 us): both keep too few warps on an SM.
#include <cooperative_groups.h>
#include <math.h>
#include <math_constants.h>
#include <string.h>

#include <atomic>

#include "cstr_internal.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxCluster = 16;
constexpr float kLn2 = 0.693147180559945309f;

struct MaskDesc {
    const uint32_t *mask;
    long long ldw;
    int n_states;
};

struct LossParams {
    MaskDesc tab[CSTR_MAX_TABLES];
    int n_tables;
    const int32_t *row_table, *states, *actions;
    const void *logits;
    void *dlogits;
    long long ld;
    int V, rows;
    float c, inv_temp;           // log2(e) / temperature, 1 / temperature
    const float *old_logp, *ref_logp, *adv, *weight;
    float lo, hi, kl;            // clip bounds of the ratio, KL coefficient
    float *loss, *logp;
    unsigned long long *oob;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    unsigned u;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
    return u;
}

// One logit.
template <bool BF16> __device__ __forceinline__ float load_one(const char *row, int tok)
{
    return BF16 ? __uint_as_float((unsigned)((const unsigned short *)row)[tok] << 16) : ((const float *)row)[tok];
}
template <bool BF16> __device__ __forceinline__ void store_one(char *row, int tok, float x)
{
    if (BF16)
        ((unsigned short *)row)[tok] = (unsigned short)pack_bf16(x, 0.f);
    else
        ((float *)row)[tok] = x;
}

// 16 bytes of logits, widened to fp32; disallowed ones (bit e of `bits` clear) become -infinity.
template <bool BF16> struct Vec {
    static constexpr int N = BF16 ? 8 : 4;
    static __device__ __forceinline__ void widen(float (&x)[N], uint4 u, unsigned bits)
    {
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float f = BF16 ? __uint_as_float(i & 1 ? w[i / 2 % 4] & 0xffff0000u : w[i / 2 % 4] << 16) : __uint_as_float(w[i % 4]);
            x[i] = (bits >> i) & 1u ? f : -CUDART_INF_F;
        }
    }
    static __device__ __forceinline__ uint4 narrow(const float (&d)[N])
    {
        if (BF16)
            return make_uint4(pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]), pack_bf16(d[4 % N], d[5 % N]), pack_bf16(d[6 % N], d[7 % N]));
        return make_uint4(__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3]));
    }
};

// x = 2^(c (x - ref)), two logits per instruction but for the exponential itself (512 x 256,000 fp32
// 242.1 us, one by one 243.6; 2,048 x 32,000 bf16 69.7 / 70.1)
template <int CNT> __device__ __forceinline__ void exponentials(float (&x)[CNT], float ref, float c)
{
    if (CNT == 1) {
        x[0] = exp2_fast((x[0] - ref) * c);
        return;
    }
#pragma unroll
    for (int i = 0; i + 1 < CNT; i += 2) {
        asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %2};\nadd.rn.f32x2 a, a, b;\n"
            "mov.b64 b, {%3, %3};\nmul.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}\n"
            : "+f"(x[i]), "+f"(x[i + 1]) : "f"(-ref), "f"(c));
        x[i] = exp2_fast(x[i]);
        x[i + 1] = exp2_fast(x[i + 1]);
    }
}

struct MaxSum {
    float m, s;
};

// Replaces CNT logits by their exponentials, counted from the running maximum, and adds them to r;
// `top`: their maximum
template <int CNT> __device__ __forceinline__ void accumulate(MaxSum &r, float (&x)[CNT], float top, float c)
{
    if (top > r.m) {
        r.s *= exp2_fast((r.m - top) * c);
        r.m = top;
    }
    const float ref = r.m == -CUDART_INF_F ? 0.f : r.m;      // (+infinity: NaN comes of it)
    float sum[2] = {r.s, 0.f};
    exponentials(x, ref, c);
#pragma unroll
    for (int i = 0; i < CNT; ++i)
        sum[i & 1] += x[i];
    r.s = sum[0] + sum[1];
}

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c)
{
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    const float ref = r.m == -CUDART_INF_F ? 0.f : r.m;
    r.s = a.s * exp2_fast((a.m - ref) * c) + b.s * exp2_fast((b.m - ref) * c);
    return r;
}

// Row scalars of the loss, by one thread: everything that the second pass needs.
struct RowResult {
    float hot, coef, loss, logp;     // gradient: d = hot [v = a] + coef 2^(c (x - m))
};

__device__ __forceinline__ RowResult row_result(const LossParams &p, bool valid, float x_a, MaxSum all, float old_logp,
                                                float ref_logp, float adv, float w)
{
    RowResult r = {0.f, 0.f, 0.f, -CUDART_INF_F};
    if (valid && x_a != -CUDART_INF_F) {
        r.logp = ((x_a - all.m) * p.c - log2f(all.s)) * kLn2;
        if (w != 0.f) {
            const float ratio = expf(r.logp - old_logp);
            // a NaN ratio stays one (fminf and fmaxf would drop it)
            const float held = ratio != ratio ? ratio : fminf(fmaxf(ratio, p.lo), p.hi);
            const float plain = ratio * adv, clipped = held * adv;
            r.loss = plain > clipped ? -clipped : -plain;
            float g = plain > clipped ? 0.f : -plain;
            if (p.ref_logp) {
                // exp(diff) - 1 as one function: near the reference policy the term is about diff^2 / 2
                const float diff = ref_logp - r.logp, k1 = expm1f(diff);
                r.loss += p.kl * (k1 - diff);
                g -= p.kl * k1;
            }
            r.loss *= w;
            r.hot = g * w * p.inv_temp;
            r.coef = r.hot == 0.f ? 0.f : -r.hot / all.s;
        }
    }
    return r;
}

// The row's automaton state's mask (null: all allowed), and whether the action is one of it.
__device__ __forceinline__ bool row_mask(const LossParams &p, int row, int a, const uint32_t *&mrow)
{
    mrow = nullptr;
    bool valid = a >= 0 && a < p.V;
    if (p.n_tables > 0) {
        const int t = p.row_table ? p.row_table[row] : 0, q = p.states[row];
        const bool known = t >= 0 && t < p.n_tables && q >= 0 && q < p.tab[t >= 0 && t < p.n_tables ? t : 0].n_states;
        if (known)
            mrow = p.tab[t].mask + (long long)q * p.tab[t].ldw;
        valid = valid && known && ((mrow[a >> 5] >> (a & 31)) & 1u);
    }
    return valid;
}

// The 16-byte vectors begin at the row's first aligned token; the tokens before and after them ("edge",
// at most 2 (N - 1)) belong to the first threads of the first CTA.  WIDE is false where the rows of the
// two buffers do not share their alignment: then every token is an edge token, dealt out over all threads.
// kUnroll: vectors of a thread in flight; 2 where the logits are only read (300 x 128,256 fp32 36.1 us,
// 4.3 TB/s; with one about 5 us more), 1 with a gradient (2,048 x 32,000 bf16, two: 6 us more, registers).
template <bool BF16, bool WIDE, int kUnroll>
__global__ void __launch_bounds__(kThreads, 8)
policy_loss_kernel(const __grid_constant__ LossParams p)
{
    using V = Vec<BF16>;
    constexpr int N = V::N, ESZ = BF16 ? 2 : 4, kWarps = kThreads / 32;
    __shared__ MaxSum s_warp[kWarps];
    __shared__ MaxSum s_part[kMaxCluster];       // every CTA's, written by its owner
    __shared__ float s_row[6];                   // old_logp, ref_logp, advantage, weight, action's logit, valid
    __shared__ float s_result[3];                // hot, coef, maximum
    cstr_wait_for_earlier_kernels();
    cstr_let_next_kernel_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int size = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    if (size > 1)                                // this CTA runs: its shared memory may be written from now on
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / size;
    const char *x_row = (const char *)p.logits + (long long)row * p.ld * ESZ;
    const int head = WIDE ? min((int)((16u - (unsigned)((uintptr_t)x_row & 15u)) & 15u) / ESZ, p.V) : p.V;
    const int vectors = WIDE ? (p.V - head) / N : 0, per = (vectors + size - 1) / size;
    const int v0 = min(part * per, vectors), v1 = min(v0 + per, vectors);
    const int edge = p.V - vectors * N;
    const int edge0 = WIDE ? (part == 0 ? tid : edge) : part * kThreads + tid, edge_step = size * kThreads;
    auto edge_token = [&](int i) { return i < head ? i : vectors * N + i; };
    const uint4 *x_vec = reinterpret_cast<const uint4 *>(x_row + head * ESZ);

    // The last warp fetches what the row's loss takes, its chain of loads (action, state, mask word,
    // logit) beside the others' first pass.
    const uint32_t *mrow;
    if (warp == kWarps - 1) {
        const int a = p.actions[row];
        const float value = lane == 0 ? p.old_logp[row] : lane == 1 ? (p.ref_logp ? p.ref_logp[row] : 0.f)
                          : lane == 2 ? p.adv[row] : lane == 3 ? (p.weight ? p.weight[row] : 1.f) : 0.f;
        const bool valid = row_mask(p, row, a, mrow);
        const float x_a = valid && lane == 4 ? load_one<BF16>(x_row, a) : 0.f;
        if (lane < 6)
            s_row[lane] = lane < 4 ? value : lane == 4 ? x_a : valid ? 1.f : 0.f;
    } else
        row_mask(p, row, 0, mrow);
    auto allowed = [&](int tok) { return !mrow || ((mrow[tok >> 5] >> (tok & 31)) & 1u); };
    // allowed bits of vector v (its tokens lie in two words where head is not a multiple of N)
    auto bits_of = [&](int v) {
        if (!mrow)
            return 0xffffffffu;
        const int tok = head + v * N;
        const unsigned lo = __ldg(mrow + (tok >> 5));
        return __funnelshift_r(lo, (tok & 31) + N > 32 ? __ldg(mrow + (tok >> 5) + 1) : 0u, tok & 31);
    };

    MaxSum r = {-CUDART_INF_F, 0.f};
#pragma unroll 1
    for (int v = v0 + tid; v < v1; v += kUnroll * kThreads) {
        uint4 raw[kUnroll];
        unsigned bits[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            bits[u] = 0u;
            raw[u] = make_uint4(0u, 0u, 0u, 0u);
            if (v + u * kThreads < v1) {
                raw[u] = x_vec[v + u * kThreads];
                bits[u] = bits_of(v + u * kThreads);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float x[N], top = -CUDART_INF_F;
            V::widen(x, raw[u], bits[u]);
#pragma unroll
            for (int i = 0; i < N; i += 2)
                top = max3(top, x[i], x[i + 1]);
            accumulate(r, x, top, p.c);
        }
    }
    for (int i = edge0; i < edge; i += edge_step) {
        const int tok = edge_token(i);
        float x[1] = {allowed(tok) ? load_one<BF16>(x_row, tok) : -CUDART_INF_F};
        accumulate(r, x, fmaxf(x[0], -CUDART_INF_F), p.c);
    }
    auto join_lanes = [&](MaxSum m) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const MaxSum o = {__shfl_xor_sync(0xffffffffu, m.m, off), __shfl_xor_sync(0xffffffffu, m.s, off)};
            m = join(m, o, p.c);
        }
        return m;
    };
    const MaxSum none = {-CUDART_INF_F, 0.f};
    r = join_lanes(r);
    if (lane == 0)
        s_warp[warp] = r;
    __syncthreads();
    if (size > 1)                                // the others run, too (they said so before their first pass)
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (warp == 0 && size > 1) {
        r = join_lanes(lane < kWarps ? s_warp[lane] : none);
        if (lane < size)                         // to every CTA; after the barrier nobody reads remotely
            *cluster.map_shared_rank(&s_part[part], lane) = r;
    }
    if (size > 1)
        cluster.sync();
    if (warp == 0) {
        const MaxSum all = join_lanes(size > 1 ? (lane < size ? s_part[lane] : none) : (lane < kWarps ? s_warp[lane] : none));
        if (lane == 0) {
            const RowResult res = row_result(p, s_row[5] != 0.f, s_row[4], all, s_row[0], s_row[1], s_row[2], s_row[3]);
            s_result[0] = res.hot;
            s_result[1] = res.coef;
            s_result[2] = all.m;
            if (part == 0) {
                p.loss[row] = res.loss;
                p.logp[row] = res.logp;
            }
        }
    }
    if (!p.dlogits)
        return;
    __syncthreads();
    char *d_row = (char *)p.dlogits + (long long)row * p.ld * ESZ;
    uint4 *d_vec = reinterpret_cast<uint4 *>(d_row + head * ESZ);
    const float hot = s_result[0], coef = s_result[1], top = s_result[2];
    if (coef == 0.f) {                           // (NaN takes another branch)
        for (int v = v0 + tid; v < v1; v += kThreads)
            __stcs(d_vec + v, make_uint4(0u, 0u, 0u, 0u));
        for (int i = edge0; i < edge; i += edge_step)
            store_one<BF16>(d_row, edge_token(i), 0.f);
        return;
    }
    const int a = p.actions[row];
    // a disallowed logit is -infinity here: its exponential and with it its gradient are 0 - unless
    // the coefficient or the maximum is not finite, which takes the second form
    const bool plain = fabsf(coef) < CUDART_INF_F && fabsf(top) < CUDART_INF_F;
#pragma unroll 1
    for (int v = v0 + tid; v < v1; v += kUnroll * kThreads) {
        uint4 raw[kUnroll];
        unsigned bits[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            bits[u] = 0u;
            raw[u] = make_uint4(0u, 0u, 0u, 0u);
            if (v + u * kThreads < v1) {
                raw[u] = __ldcs(x_vec + v + u * kThreads);
                bits[u] = bits_of(v + u * kThreads);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float x[N];
            V::widen(x, raw[u], bits[u]);
            if (plain) {
                exponentials(x, top, p.c);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[i] *= coef;
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[i] = (bits[u] >> i) & 1u ? coef * exp2_fast((x[i] - top) * p.c) : 0.f;
            }
            const int at = a - (head + (v + u * kThreads) * N);      // the action among the vector's tokens
            if ((unsigned)at < (unsigned)N) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[i] += at == i ? hot : 0.f;
            }
            if (v + u * kThreads < v1)
                __stcs(d_vec + v + u * kThreads, V::narrow(x));
        }
    }
    for (int i = edge0; i < edge; i += edge_step) {
        const int tok = edge_token(i);
        float d = allowed(tok) ? coef * exp2_fast((load_one<BF16>(x_row, tok) - top) * p.c) : 0.f;
        if (tok == a)
            d += hot;
        store_one<BF16>(d_row, tok, d);
    }
}

int launch(void (*kernel)(LossParams), const LossParams &p, int size, cudaStream_t stream)
{
    if (size > 8)
        CSTR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    return cstr_launch(kernel, (long long)p.rows * size, kThreads, size, 0, stream, p);
}

}  // namespace

extern "C" int cstr_policy_loss(const cstr_table_t *const *tables, int32_t n_tables,
                                const int32_t *row_table, const int32_t *states, const void *logits,
                                int32_t dtype, int64_t ld, int32_t vocab_size, float temperature,
                                const int32_t *actions, const float *old_logp, const float *ref_logp,
                                const float *advantages, const float *weight, float clip_low,
                                float clip_high, float kl_coef, float *loss_out, float *logp_out,
                                void *dlogits, int32_t rows, void *cuda_stream)
{
    if (n_tables < 0 || n_tables > CSTR_MAX_TABLES)
        return cstr_fail(CSTR_ERR_ARG, "cstr_policy_loss: n_tables = %d, need 0..%d", n_tables,
                         CSTR_MAX_TABLES);
    if (dtype != CSTR_F32 && dtype != CSTR_BF16)
        return cstr_fail(CSTR_ERR_DTYPE, "cstr_policy_loss: unknown dtype %d", dtype);
    if (rows < 0 || vocab_size < 1)
        return cstr_fail(CSTR_ERR_ARG, "cstr_policy_loss: rows = %d, vocab_size = %d", rows, vocab_size);
    const float scale_log2 = (float)(1.4426950408889634 / temperature);
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(scale_log2) || !(clip_low >= 0.f) || !(clip_high >= 0.f) ||
        !isfinite(kl_coef))
        return cstr_fail(CSTR_ERR_ARG, "cstr_policy_loss: temperature = %g, clip = %g / %g, kl = %g",
                         temperature, clip_low, clip_high, kl_coef);
    if (ld < vocab_size)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_policy_loss: ld = %lld is below V = %d", (long long)ld,
                         vocab_size);
    if (rows == 0)
        return CSTR_OK;
    if (!logits || !actions || !old_logp || !advantages || !loss_out || !logp_out ||
        (n_tables > 0 && (!tables || !states)))
        return cstr_fail(CSTR_ERR_NULL, "cstr_policy_loss: null pointer");
    const uintptr_t element = dtype == CSTR_BF16 ? 2 : 4;
    if ((uintptr_t)logits % element || (uintptr_t)dlogits % element)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_policy_loss: logits and dlogits must start on whole elements");
    int device = -1;
    CSTR_CUDA_TRY(cudaGetDevice(&device));
    LossParams p;
    memset(&p, 0, sizeof p);
    for (int32_t i = 0; i < n_tables; ++i) {
        const cstr_table *t = tables[i];
        if (!t)
            return cstr_fail(CSTR_ERR_NULL, "cstr_policy_loss: tables[%d] is null", i);
        if (t->device != device)
            return cstr_fail(CSTR_ERR_DEVICE, "cstr_policy_loss: tables[%d] is on device %d, device %d is "
                             "current", i, t->device, device);
        if (t->n_states < 1)
            return cstr_fail(CSTR_ERR_ARG, "cstr_policy_loss: tables[%d] has not been built", i);
        if (t->V != vocab_size)
            return cstr_fail(CSTR_ERR_SHAPE, "cstr_policy_loss: tables[%d] has V = %d, vocab_size is %d", i,
                             t->V, vocab_size);
        p.tab[i].mask = t->mask;
        p.tab[i].ldw = t->ldw;
        p.tab[i].n_states = t->n_states;
    }
    p.n_tables = n_tables;
    p.row_table = row_table;
    p.states = states;
    p.actions = actions;
    p.logits = logits;
    p.dlogits = dlogits;
    p.ld = ld;
    p.V = vocab_size;
    p.rows = rows;
    p.c = scale_log2;
    p.inv_temp = 1.f / temperature;
    p.old_logp = old_logp;
    p.ref_logp = ref_logp;
    p.adv = advantages;
    p.weight = weight;
    p.lo = 1.f - clip_low;
    p.hi = 1.f + clip_high;
    p.kl = kl_coef;
    p.loss = loss_out;
    p.logp = logp_out;
    p.oob = CSTR_OOB_RECORD();
    const bool bf16 = dtype == CSTR_BF16;
    if ((long long)rows * kMaxCluster > 0x7fffffffLL)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_policy_loss: rows x vocabulary too large for one launch");
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    // rows of both buffers begin at the same place of their 16 bytes
    const bool together = !dlogits || (((uintptr_t)logits ^ (uintptr_t)dlogits) & 15u) == 0;
    // 64 KB of a row per CTA; smaller shares, down to 2,048 tokens, while there are fewer CTAs than
    // two per SM (4 x 32,000 fp32 6.5 us, unshared 13.5 us; 16 x 128,256 11.9 / 18.8 us)
    static std::atomic<int> known[64];
    int sms = device >= 0 && device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
    if (sms == 0) {
        CSTR_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
        if (device >= 0 && device < 64)
            known[device].store(sms, std::memory_order_relaxed);
    }
    const long long share = bf16 ? 32768 : 16384;
    int size = 1;
    while (size < kMaxCluster && (vocab_size > share * size ||
                                  (rows * (long long)size <= sms && vocab_size >= 4096LL * size)))
        size *= 2;
    void (*kernel)(LossParams);
    if (!together)
        kernel = bf16 ? policy_loss_kernel<true, false, 1> : policy_loss_kernel<false, false, 1>;
    else if (dlogits)
        kernel = bf16 ? policy_loss_kernel<true, true, 1> : policy_loss_kernel<false, true, 1>;
    else
        kernel = bf16 ? policy_loss_kernel<true, true, 2> : policy_loss_kernel<false, true, 2>;
    return launch(kernel, p, size, stream);
}
