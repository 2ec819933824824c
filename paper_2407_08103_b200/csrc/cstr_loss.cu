// Clipped policy loss with a KL term over the constrained distribution, forward
// and gradient, in one kernel: a cluster of CTAs takes one row of logits.
//
// Mathematics, in base 2 with c = log2(e) / temperature: one pass for the running
// maximum m of the allowed logits x_v and s = sum 2^(c (x_v - m)); log2 p_a =
// c (x_a - m) - log2 s; ratio, loss and d loss / d logp from that; a second pass
// for p_v = 2^(c (x_v - m)) / s.  The maximum is subtracted before the product, so
// that logits near the type's lowest value do not overflow.
//
// Bound: the row is read from memory once (the second pass finds it in the L2
// cache) and the gradient written once.
#include <cooperative_groups.h>
#include <math.h>
#include <math_constants.h>
#include <string.h>

#include "cstr_internal.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256;
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
    int V, rows, slice;          // slice: tokens per CTA of a cluster, a multiple of 32
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

// VEC consecutive logits as fp32 / back, 16 bytes at once where the layout allows it
template <bool BF16, int VEC>
__device__ __forceinline__ void load_vec(float (&x)[VEC], const void *row, int tok)
{
    if (VEC == 1) {
        x[0] = BF16 ? __uint_as_float((unsigned)((const unsigned short *)row)[tok] << 16)
                    : ((const float *)row)[tok];
        return;
    }
    const uint4 u = *reinterpret_cast<const uint4 *>((const char *)row + (long long)tok * (BF16 ? 2 : 4));
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        x[i] = BF16 ? __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16)
                    : __uint_as_float(w[i % 4]);
}

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    unsigned u;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
    return u;
}

template <bool BF16, int VEC>
__device__ __forceinline__ void store_vec(void *row, int tok, const float (&x)[VEC])
{
    if (VEC == 1) {
        if (BF16)
            ((unsigned short *)row)[tok] = (unsigned short)pack_bf16(x[0], 0.f);
        else
            ((float *)row)[tok] = x[0];
        return;
    }
    uint4 u;
    if (BF16)
        u = make_uint4(pack_bf16(x[0], x[1 % VEC]), pack_bf16(x[2 % VEC], x[3 % VEC]),
                       pack_bf16(x[4 % VEC], x[5 % VEC]), pack_bf16(x[6 % VEC], x[7 % VEC]));
    else
        u = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1 % VEC]), __float_as_uint(x[2 % VEC]),
                       __float_as_uint(x[3 % VEC]));
    __stcs(reinterpret_cast<uint4 *>((char *)row + (long long)tok * (BF16 ? 2 : 4)), u);
}

struct MaxSum {
    float m, s;
};

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c)
{
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    const float ref = r.m == -CUDART_INF_F ? 0.f : r.m;
    r.s = a.s * exp2_fast((a.m - ref) * c) + b.s * exp2_fast((b.m - ref) * c);
    return r;
}

template <bool BF16, int VEC>
__global__ void __launch_bounds__(kThreads)
policy_loss_kernel(const __grid_constant__ LossParams p)
{
    __shared__ MaxSum s_warp[kThreads / 32];
    __shared__ MaxSum s_cta;
    __shared__ float s_coef[2];                  // gradient: d = coef[0] [v = a] + coef[1] 2^(c (x - m))
    __shared__ float s_top;
    cg::cluster_group cluster = cg::this_cluster();
    const int size = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / size;
    const long long at = (long long)row * p.ld * (BF16 ? 2 : 4);
    const void *x_row = (const char *)p.logits + at;
    const int a = p.actions[row];

    const uint32_t *mrow = nullptr;
    bool valid = a >= 0 && a < p.V;
    if (p.n_tables > 0) {
        const int t = p.row_table ? p.row_table[row] : 0, q = p.states[row];
        const bool known = t >= 0 && t < p.n_tables && q >= 0 && q < p.tab[t >= 0 && t < p.n_tables ? t : 0].n_states;
        if (known)
            mrow = p.tab[t].mask + (long long)q * p.tab[t].ldw;
        valid = valid && known && ((mrow[a >> 5] >> (a & 31)) & 1u);
    }
    const int begin = min(part * p.slice, p.V), end = min(begin + p.slice, p.V);

    MaxSum r = {-CUDART_INF_F, 0.f};
    float x_a = 0.f;
    if (valid) {
        float one[1];
        load_vec<BF16, 1>(one, x_row, a);
        x_a = one[0];
        for (int tok = begin + tid * VEC; tok < end; tok += kThreads * VEC) {
            float x[VEC];
            load_vec<BF16, VEC>(x, x_row, tok);
            const unsigned bits = mrow ? __ldg(mrow + (tok >> 5)) >> (tok & 31) : 0xffffffffu;
            float top = -CUDART_INF_F;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                x[i] = (bits >> i) & 1u ? x[i] : -CUDART_INF_F;
                top = fmaxf(top, x[i]);
            }
            if (top > r.m) {
                r.s *= exp2_fast((r.m - top) * p.c);
                r.m = top;
            }
            const float ref = r.m == -CUDART_INF_F ? 0.f : r.m;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                r.s += exp2_fast((x[i] - ref) * p.c);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const MaxSum o = {__shfl_xor_sync(0xffffffffu, r.m, off), __shfl_xor_sync(0xffffffffu, r.s, off)};
            r = join(r, o, p.c);
        }
        if (lane == 0)
            s_warp[warp] = r;
    }
    __syncthreads();
    if (tid == 0) {
        if (valid)
            for (int w = 1; w < kThreads / 32; ++w)
                r = join(r, s_warp[w], p.c);
        s_cta = r;
    }
    if (size > 1)
        cluster.sync();
    if (tid == 0) {
        MaxSum all = {-CUDART_INF_F, 0.f};
        if (valid)
            for (int c = 0; c < size; ++c)
                all = join(all, *cluster.map_shared_rank(&s_cta, c), p.c);
        float loss = 0.f, logp = -CUDART_INF_F, g = 0.f;
        const float w = p.weight ? p.weight[row] : 1.f;
        const float log2p = (x_a - all.m) * p.c - log2f(all.s);
        if (valid && x_a != -CUDART_INF_F) {
            logp = log2p * kLn2;
            if (w != 0.f) {
                const float ratio = expf(logp - p.old_logp[row]), adv = p.adv[row];
                // a NaN ratio stays one (fminf and fmaxf would drop it)
                const float held = ratio != ratio ? ratio : fminf(fmaxf(ratio, p.lo), p.hi);
                const float plain = ratio * adv, clipped = held * adv;
                loss = plain > clipped ? -clipped : -plain;
                g = plain > clipped ? 0.f : -plain;
                if (p.ref_logp) {
                    const float diff = p.ref_logp[row] - logp, k = expf(diff);
                    loss += p.kl * (k - diff - 1.f);
                    g += p.kl * (1.f - k);
                }
                loss *= w;
                g *= w * p.inv_temp;
            }
        }
        s_coef[0] = g;
        s_coef[1] = g == 0.f ? 0.f : -g / all.s;
        s_top = all.m;
        if (part == 0) {
            p.loss[row] = loss;
            p.logp[row] = logp;
        }
    }
    if (size > 1)
        cluster.sync();                          // nobody leaves while s_cta is read
    else
        __syncthreads();
    if (!p.dlogits)
        return;
    void *d_row = (char *)p.dlogits + at;
    const float hot = s_coef[0], coef = s_coef[1], top = s_top;
    if (coef == 0.f) {                           // (NaN takes the other branch)
        const float zero[VEC] = {};
        for (int tok = begin + tid * VEC; tok < end; tok += kThreads * VEC)
            store_vec<BF16, VEC>(d_row, tok, zero);
        return;
    }
    for (int tok = begin + tid * VEC; tok < end; tok += kThreads * VEC) {
        float x[VEC];
        load_vec<BF16, VEC>(x, x_row, tok);
        const unsigned bits = mrow ? __ldg(mrow + (tok >> 5)) >> (tok & 31) : 0xffffffffu;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            x[i] = (bits >> i) & 1u ? coef * exp2_fast((x[i] - top) * p.c) : 0.f;
            if (tok + i == a)
                x[i] += hot;
        }
        store_vec<BF16, VEC>(d_row, tok, x);
    }
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

template <bool BF16, int VEC>
int launch(const LossParams &p, int size, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)((long long)p.rows * size));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CSTR_CUDA_TRY(cudaLaunchKernelEx(&cfg, policy_loss_kernel<BF16, VEC>, p));
    return CSTR_OK;
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
    if (!(temperature > 0.f) || !isfinite(temperature) || !(clip_low >= 0.f) || !(clip_high >= 0.f) ||
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
    p.c = (float)(1.4426950408889634 / temperature);
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
    const int vec = bf16 ? 8 : 4;
    int size = 1;
    while (size < 8 && (long long)vocab_size > 8192LL * size)
        size *= 2;
    if ((long long)rows * size > 0x7fffffffLL)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_policy_loss: rows x vocabulary too large for one launch");
    p.slice = (int)((((long long)vocab_size + size - 1) / size + 31) / 32 * 32);
    const bool wide = aligned16(logits) && (!dlogits || aligned16(dlogits)) && vocab_size % vec == 0 &&
                      (ld * (bf16 ? 2 : 4)) % 16 == 0;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (bf16)
        return wide ? launch<true, 8>(p, size, stream) : launch<true, 1>(p, size, stream);
    return wide ? launch<false, 4>(p, size, stream) : launch<false, 1>(p, size, stream);
}
