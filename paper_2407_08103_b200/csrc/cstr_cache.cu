// Key / value cache of a batch with a shared prompt: handle, argument checks,
// and the insertion of new tokens with eviction by accumulated attention weight.
#include <math.h>
#include <string.h>

#include <new>

#include "cstr_cache.cuh"

namespace {

// ---- insertion -------------------------------------------------------------
//
// One CTA per row and key / value head.  Entries are ordered by (protected,
// weight, slot).  Their 32-bit keys (order-preserving bits of the weight;
// all ones when protected; 0 for NaN) are read once into shared memory; the
// e-th smallest key is found by four passes over 8-bit digits, counting into
// 256 bins, and ties at that key are taken in slot order.  Evicted slots below
// the new length and surviving slots past it are then enumerated in slot order
// by ballots and prefix sums, and the i-th free place gets the i-th mover.  All
// of it is counting, so the result does not depend on the order of atomics.
//
// Bound: 8 bytes per entry (weight, age) are read; only new tokens, and
// survivors past the new length, are copied.
constexpr int kInsertThreads = 256;

struct InsertParams {
    const char *k_new, *v_new;
    long long nk_sb, nk_st, nk_sh, nv_sb, nv_st, nv_sh;
    char *ck, *cv;
    long long ck_sb, ck_ss, ck_sh, cv_sb, cv_ss, cv_sh;
    float *weight;
    int32_t *age, *lens;
    const int32_t *n_new, *pos;
    unsigned int *ticket;
    int32_t *list;       // null: keys and places live in shared memory
    int B, Hk, D, cap, T, budget, recent;
    unsigned long long *oob;
};

__device__ __forceinline__ unsigned evict_key(float w, int age, int protect_from)
{
    if (age >= protect_from)
        return 0xffffffffu;
    if (w != w)
        return 0u;
    const unsigned u = __float_as_uint(w + 0.0f);                 // -0 counts as 0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix over the block of one flag per thread; total in *all.
__device__ __forceinline__ int block_rank(bool flag, int *s_warp, int &all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned hits = __ballot_sync(0xffffffffu, flag);
    __syncthreads();                                              // s_warp free again
    if (lane == 0)
        s_warp[warp] = __popc(hits);
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kInsertThreads / 32; ++w) {
        before += w < warp ? s_warp[w] : 0;
        all += s_warp[w];
    }
    return before + __popc(hits & ((1u << lane) - 1u));
}

__global__ void __launch_bounds__(kInsertThreads)
cache_insert_kernel(const __grid_constant__ InsertParams p)
{
    extern __shared__ int s_dyn[];
    __shared__ int s_bin[256];
    __shared__ int s_warp[kInsertThreads / 32];
    __shared__ int s_digit, s_below;
    const int tid = threadIdx.x;
    const int b = blockIdx.x / p.Hk, kh = blockIdx.x - b * p.Hk;
    const int len = min(max(p.lens[b], 0), p.cap);
    const int n = p.n_new ? min(max(p.n_new[b], 0), p.T) : p.T;
    const int pos = p.pos[b];
    const int new_len = min(len + n, p.budget);
    const int evict = len + n - new_len;
    const long long entry0 = ((long long)b * p.Hk + kh) * p.cap;
    float *weight = p.weight + entry0;
    int32_t *age = p.age + entry0;
    unsigned *keys = reinterpret_cast<unsigned *>(p.list ? p.list + entry0 * 2 : s_dyn);
    int *place = reinterpret_cast<int *>(keys + p.cap);           // free places, ascending
    int n_old = 0;                                                // survivors past the new length

    if (evict > 0) {
        const int protect_from = pos + n - p.recent;
        for (int j = tid; j < len; j += kInsertThreads)
            keys[j] = evict_key(weight[j], age[j], protect_from);
        unsigned prefix = 0;
        int want = evict;                                         // rank within the current prefix
#pragma unroll 1
        for (int shift = 24; shift >= 0; shift -= 8) {
            s_bin[tid] = 0;
            __syncthreads();
            for (int j = tid; j < len; j += kInsertThreads) {
                const unsigned k = keys[j];
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))
                    atomicAdd(&s_bin[(k >> shift) & 255u], 1);
            }
            __syncthreads();
            if (tid < 32) {                                       // first digit whose count reaches want
                int sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    sum += s_bin[tid * 8 + i];
                int upto = sum;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const int o = __shfl_up_sync(0xffffffffu, upto, off);
                    upto += tid >= off ? o : 0;
                }
                const unsigned reach = __ballot_sync(0xffffffffu, upto >= want);
                if (tid == __ffs((int)reach) - 1) {
                    int below = upto - sum, d = 0;
                    while (d < 7 && below + s_bin[tid * 8 + d] < want)
                        below += s_bin[tid * 8 + d++];
                    s_digit = tid * 8 + d;
                    s_below = below;
                }
            }
            __syncthreads();
            prefix |= (unsigned)s_digit << shift;
            want -= s_below;
            __syncthreads();
        }
        // evicted: key < prefix, and the first `want` slots with key == prefix.  Free places and
        // movers in slot order; movers are listed from the end of `place`.
        int ties = 0, holes = 0;
        for (int j0 = 0; j0 < len; j0 += kInsertThreads) {
            const int j = j0 + tid;
            const unsigned k = j < len ? keys[j] : 0u;
            int all;
            const int tie = block_rank(j < len && k == prefix, s_warp, all) + ties;
            const bool gone = j < len && (k < prefix || (k == prefix && tie < want));
            ties += all;
            const int hole = block_rank(gone && j < new_len, s_warp, all) + holes;
            if (gone && j < new_len)
                place[hole] = j;
            holes += all;
            if (j0 + kInsertThreads > new_len && len > new_len) {  // uniform
                const int mover = block_rank(j < len && !gone && j >= new_len, s_warp, all) + n_old;
                if (j < len && !gone && j >= new_len)
                    place[p.cap - 1 - mover] = j;
                n_old += all;
            }
        }
        for (int j = len + tid; j < new_len; j += kInsertThreads)
            place[holes + j - len] = j;
        __syncthreads();
    }

    // copies: mover i -> free place i, 16 bytes a thread
    const int moves = evict > 0 ? n_old + n : n;
    const int per = p.D / 8;                                      // 16-byte pieces of a row
    for (int i = tid; i < moves * per * 2; i += kInsertThreads) {
        const int half = i >= moves * per;                        // keys first, then values
        const int at = i - half * moves * per;
        const int mv = at / per, piece = at - mv * per;
        const int dst = evict > 0 ? place[mv] : len + mv;
        if (!CSTR_INB(p.oob, dst, p.cap, CSTR_SITE_CACHE))
            continue;
        const long long sb = half ? p.cv_sb : p.ck_sb, ss = half ? p.cv_ss : p.ck_ss,
                        sh = half ? p.cv_sh : p.ck_sh;
        char *cache = (half ? p.cv : p.ck) + ((long long)b * sb + (long long)kh * sh) * 2;
        const char *from;
        if (mv < n_old) {
            const int j = place[p.cap - 1 - mv];
            if (!CSTR_INB(p.oob, j, p.cap, CSTR_SITE_CACHE))
                continue;
            from = cache + (long long)j * ss * 2;
        } else {
            const int t = mv - n_old;
            from = half ? p.v_new + ((long long)b * p.nv_sb + (long long)t * p.nv_st + (long long)kh * p.nv_sh) * 2
                        : p.k_new + ((long long)b * p.nk_sb + (long long)t * p.nk_st + (long long)kh * p.nk_sh) * 2;
        }
        *reinterpret_cast<uint4 *>(cache + (long long)dst * ss * 2 + piece * 16) =
            *reinterpret_cast<const uint4 *>(from + piece * 16);
    }
    for (int mv = tid; mv < moves; mv += kInsertThreads) {
        const int dst = evict > 0 ? place[mv] : len + mv;
        if (!CSTR_INB(p.oob, dst, p.cap, CSTR_SITE_CACHE))
            continue;
        if (mv < n_old) {
            const int j = place[p.cap - 1 - mv];
            weight[dst] = weight[j];
            age[dst] = age[j];
        } else {
            weight[dst] = 0.f;
            age[dst] = pos + mv - n_old;
        }
    }

    // every CTA of the row has read lens[b] when it arrives here; the last one replaces it
    __syncthreads();
    if (tid == 0) {
        const unsigned prev = atomicAdd(p.ticket + b, 1u);
        if (prev == (unsigned)p.Hk - 1u) {
            p.ticket[b] = 0u;
            p.lens[b] = new_len;
        }
    }
}

int strides_ok(const char *what, const int64_t *s, int n)
{
    for (int i = 0; i < n; ++i)
        if (s[i] % 8)
            return cstr_fail(CSTR_ERR_SHAPE, "%s: stride %lld is no multiple of 8 elements", what,
                             (long long)s[i]);
    return CSTR_OK;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace

int cstr_launch_insert(const cstr_cache &c, const cstr_insert_args &a, cudaStream_t stream)
{
    InsertParams p;
    memset(&p, 0, sizeof p);
    p.k_new = (const char *)a.k_new;
    p.v_new = (const char *)a.v_new;
    p.nk_sb = a.k_sb, p.nk_st = a.k_st, p.nk_sh = a.k_sh;
    p.nv_sb = a.v_sb, p.nv_st = a.v_st, p.nv_sh = a.v_sh;
    p.ck = (char *)c.cache_k;
    p.cv = (char *)c.cache_v;
    p.ck_sb = c.ck_sb, p.ck_ss = c.ck_ss, p.ck_sh = c.ck_sh;
    p.cv_sb = c.cv_sb, p.cv_ss = c.cv_ss, p.cv_sh = c.cv_sh;
    p.weight = c.weight;
    p.age = c.age;
    p.lens = c.lens;
    p.n_new = a.n_new;
    p.pos = a.pos;
    p.ticket = c.ticket;
    p.list = c.list;
    p.B = c.batch;
    p.Hk = c.n_kv_heads;
    p.D = c.head_dim;
    p.cap = c.cap;
    p.T = a.tokens;
    p.budget = a.budget;
    p.recent = a.recent;
    p.oob = CSTR_OOB_RECORD();
    const int smem = c.list ? 0 : c.cap * 8;
    if (smem > 48 * 1024)
        CSTR_CUDA_TRY(cudaFuncSetAttribute(cache_insert_kernel,
                                           cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    cache_insert_kernel<<<(unsigned)(c.batch * c.n_kv_heads), kInsertThreads, smem, stream>>>(p);
    CSTR_CUDA_TRY(cudaGetLastError());
    return CSTR_OK;
}

extern "C" void cstr_free_cache(cstr_cache_t *c)
{
    if (!c)
        return;
    cudaFree(c->ticket);
    cudaFree(c->list);
    cudaFree(c->part_o);
    cudaFree(c->part_ml);
    cudaFree(c->status);
    delete c;
}

extern "C" int cstr_cache_create(int32_t dtype, int32_t batch, int32_t n_heads, int32_t n_kv_heads,
                                 int32_t head_dim, int32_t max_tokens, const void *prefix_k,
                                 const void *prefix_v, int64_t prefix_len,
                                 const int64_t *prefix_strides, void *cache_k, void *cache_v,
                                 int32_t cap, const int64_t *cache_strides, float *weight,
                                 int32_t *age, int32_t *lens, cstr_cache_t **out)
{
    if (!out)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_create: null pointer");
    *out = nullptr;
    if (!cache_k || !cache_v || !cache_strides || !lens ||
        (prefix_len > 0 && (!prefix_k || !prefix_v || !prefix_strides)))
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_create: null pointer");
    if (dtype != CSTR_BF16 && dtype != CSTR_F16)
        return cstr_fail(CSTR_ERR_DTYPE, "cstr_cache_create: dtype %d is neither bf16 nor f16", dtype);
    if (batch < 1 || n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads)
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_create: batch = %d, heads = %d, kv heads = %d", batch,
                         n_heads, n_kv_heads);
    if (head_dim < 8 || head_dim > 128 || head_dim % 8)
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_create: head_dim = %d, need a multiple of 8 in 8..128",
                         head_dim);
    if (max_tokens < 1 || cap < 1 || prefix_len < 0)
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_create: max_tokens = %d, cap = %d, prefix_len = %lld",
                         max_tokens, cap, (long long)prefix_len);
    // indices of one row's key list, and of a call's query rows, are 32-bit
    if (prefix_len + cap > 0x3fffffffLL || (int64_t)batch * n_kv_heads > 0x0fffffffLL ||
        (int64_t)max_tokens * n_heads > 0x00ffffffLL)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_cache_create: too large (keys a row %lld, rows x heads %lld, "
                         "tokens x heads %lld)", (long long)(prefix_len + cap),
                         (long long)batch * n_kv_heads, (long long)max_tokens * n_heads);
    int rc = strides_ok("cstr_cache_create", cache_strides, 6);
    if (!rc && prefix_len > 0)
        rc = strides_ok("cstr_cache_create", prefix_strides, 4);
    if (rc)
        return rc;
    if (!aligned16(cache_k) || !aligned16(cache_v) ||
        (prefix_len > 0 && (!aligned16(prefix_k) || !aligned16(prefix_v))))
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_cache_create: keys and values must start on 16 bytes");
    cstr_cache *c = new (std::nothrow) cstr_cache();
    if (!c)
        return cstr_fail(CSTR_ERR_NOMEM, "cstr_cache_create: out of host memory");
    memset(c, 0, sizeof *c);
    c->dtype = dtype;
    c->batch = batch;
    c->n_heads = n_heads;
    c->n_kv_heads = n_kv_heads;
    c->head_dim = head_dim;
    c->max_tokens = max_tokens;
    c->cap = cap;
    c->prefix_len = prefix_len;
    if (prefix_len > 0) {
        c->prefix_k = prefix_k;
        c->prefix_v = prefix_v;
        c->pk_st = prefix_strides[0], c->pk_sh = prefix_strides[1];
        c->pv_st = prefix_strides[2], c->pv_sh = prefix_strides[3];
    }
    c->cache_k = cache_k;
    c->cache_v = cache_v;
    c->ck_sb = cache_strides[0], c->ck_ss = cache_strides[1], c->ck_sh = cache_strides[2];
    c->cv_sb = cache_strides[3], c->cv_ss = cache_strides[4], c->cv_sh = cache_strides[5];
    c->weight = weight;
    c->age = age;
    c->lens = lens;
    cudaError_t e = cudaGetDevice(&c->device);
    if (e == cudaSuccess)
        e = cudaDeviceGetAttribute(&c->sm_count, cudaDevAttrMultiProcessorCount, c->device);
    if (e == cudaSuccess)
        e = cudaMalloc((void **)&c->ticket, (size_t)batch * 4);
    if (e == cudaSuccess)
        e = cudaMemset(c->ticket, 0, (size_t)batch * 4);
    if (e == cudaSuccess)
        e = cudaMalloc((void **)&c->status, 4);
    if (e == cudaSuccess)
        e = cudaMemset(c->status, 0, 4);
    if (e == cudaSuccess && cap > CSTR_INSERT_SMEM_SLOTS && weight && age)
        e = cudaMalloc((void **)&c->list, (size_t)batch * n_kv_heads * cap * 8);
    if (e != cudaSuccess) {
        rc = cstr_fail(e == cudaErrorMemoryAllocation ? CSTR_ERR_NOMEM : CSTR_ERR_CUDA,
                       "cstr_cache_create: %s", cudaGetErrorString(e));
        cstr_free_cache(c);
        return rc;
    }
    if (prefix_len > 0) {
        rc = cstr_prefix_init(c);
        if (rc) {
            cstr_free_cache(c);
            return rc;
        }
    }
    *out = c;
    return CSTR_OK;
}

extern "C" int cstr_cache_insert(cstr_cache_t *c, const void *k_new, const void *v_new,
                                 const int64_t *new_strides, int32_t n_tokens, const int32_t *n_new,
                                 const int32_t *pos, int32_t budget, int32_t recent, void *cuda_stream)
{
    if (!c || !pos || (n_tokens > 0 && (!k_new || !v_new || !new_strides)))
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_insert: null pointer");
    if (!c->weight || !c->age)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_insert: the cache was created without weight or age");
    if (budget < 1 || budget > c->cap || recent < 0 || recent > budget)
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_insert: budget = %d (cap %d), recent = %d", budget,
                         c->cap, recent);
    if (n_tokens < 0 || n_tokens > c->max_tokens || n_tokens > budget)
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_insert: n_tokens = %d, need 0..%d", n_tokens,
                         c->max_tokens < budget ? c->max_tokens : budget);
    cstr_insert_args a;
    memset(&a, 0, sizeof a);
    if (n_tokens > 0) {
        const int rc = strides_ok("cstr_cache_insert", new_strides, 6);
        if (rc)
            return rc;
        if (!aligned16(k_new) || !aligned16(v_new))
            return cstr_fail(CSTR_ERR_SHAPE, "cstr_cache_insert: k_new and v_new must start on 16 bytes");
        a.k_sb = new_strides[0], a.k_st = new_strides[1], a.k_sh = new_strides[2];
        a.v_sb = new_strides[3], a.v_st = new_strides[4], a.v_sh = new_strides[5];
    }
    const int rc = cstr_check_device(c->device, "cache");
    if (rc)
        return rc;
    a.k_new = k_new;
    a.v_new = v_new;
    a.tokens = n_tokens;
    a.n_new = n_new;
    a.pos = pos;
    a.budget = budget;
    a.recent = recent;
    return cstr_launch_insert(*c, a, (cudaStream_t)cuda_stream);
}

extern "C" int cstr_cache_attention(cstr_cache_t *c, const void *q, const int64_t *q_strides,
                                    int32_t n_tokens, const int32_t *pos, const int32_t *n_query,
                                    float scale, int32_t accumulate, void *out,
                                    const int64_t *out_strides, float *lse_out, void *cuda_stream)
{
    if (!c || !q || !q_strides || !out || !out_strides)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_attention: null pointer");
    if (accumulate && !c->weight)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_attention: the cache was created without weight");
    if (pos && !c->age)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_attention: the cache was created without age");
    if (n_tokens < 1 || n_tokens > c->max_tokens)
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_attention: n_tokens = %d, need 1..%d", n_tokens,
                         c->max_tokens);
    if (!isfinite(scale))
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_attention: scale is not finite");
    int rc = strides_ok("cstr_cache_attention", q_strides, 3);
    if (!rc)
        rc = strides_ok("cstr_cache_attention", out_strides, 3);
    if (rc)
        return rc;
    if (!aligned16(q) || !aligned16(out))
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_cache_attention: q and out must start on 16 bytes");
    rc = cstr_check_device(c->device, "cache");
    if (rc)
        return rc;
    cstr_row_args a;
    memset(&a, 0, sizeof a);
    a.q = q;
    a.q_sb = q_strides[0], a.q_st = q_strides[1], a.q_sh = q_strides[2];
    a.out = out;
    a.o_sb = out_strides[0], a.o_st = out_strides[1], a.o_sh = out_strides[2];
    a.lse_out = lse_out;
    a.tokens = n_tokens;
    a.pos = pos;
    a.n_query = n_query;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.accumulate = accumulate ? 1 : 0;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const bool tensor = c->has_maps && c->prefix_len >= 128;
    if (tensor) {
        rc = cstr_launch_prefix(*c, a, stream);
        if (rc)
            return rc;
    }
    return cstr_launch_row_attention(*c, a, !tensor, stream);
}

extern "C" int cstr_cache_status(cstr_cache_t *c, void *cuda_stream, int64_t *gave_up)
{
    if (!c || !gave_up)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_status: null pointer");
    const int rc = cstr_check_device(c->device, "cache");
    if (rc)
        return rc;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    int n = 0;
    CSTR_CUDA_TRY(cudaMemcpyAsync(&n, c->status, 4, cudaMemcpyDeviceToHost, stream));
    CSTR_CUDA_TRY(cudaMemsetAsync(c->status, 0, 4, stream));
    CSTR_CUDA_TRY(cudaStreamSynchronize(stream));
    *gave_up = n;
    return CSTR_OK;
}
