// Internal definitions of the key / value cache and its attention (not part of the ABI).
#pragma once

#include <cuda_fp16.h>

#include <atomic>

#include "cstr_internal.cuh"

// Allows `kernel` its dynamic shared memory on `device`.  `most` is the largest amount that any call asks
// for, the same every time: threads that launch the kernel side by side never lower each other's limit.
// `allowed` (one array per kernel) remembers where it has been done, so that a decoding loop does not ask again.
template <typename K>
int cstr_allow_smem(K kernel, std::atomic<bool> (&allowed)[64], int device, int most)
{
    if (device >= 0 && device < 64 && allowed[device].load(std::memory_order_relaxed))
        return CSTR_OK;
    CSTR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    if (device >= 0 && device < 64)
        allowed[device].store(true, std::memory_order_relaxed);
    return CSTR_OK;
}

// Reference of an online softmax (base 2) whose probabilities enter a product in a 16-bit type.  It is set
// kBelow under the maximum and moves when a score exceeds it by more than kLag, so that most keys need no
// rescaling of the sums (the running maximum of Milakov and Gimelshein, arXiv:1805.02867, with a lag).  The
// probabilities stay below 2^kLag, in range of the type.  Half precision has few bits below 2^-14 and none
// below 2^-24: lifting its probabilities by 2^7 keeps all bits down to 2^-21 of the largest one.
template <typename T> struct cstr_softmax_reference {
    static constexpr float kBelow = 0.f, kLag = 8.f;          // bfloat16: the exponents of fp32
};
template <> struct cstr_softmax_reference<__half> {
    static constexpr float kBelow = 7.f, kLag = 15.f;
};

// What cstr_cache_create recorded: caller-owned arrays and their strides (in
// elements), and the scratch that the handle's calls share.
struct cstr_cache {
    int device;
    int32_t sm_count;
    int32_t dtype, batch, n_heads, n_kv_heads, head_dim, max_tokens, cap;
    int64_t prefix_len;
    const void *prefix_k, *prefix_v;
    int64_t pk_st, pk_sh, pv_st, pv_sh;                   // token, head
    void *cache_k, *cache_v;
    int64_t ck_sb, ck_ss, ck_sh, cv_sb, cv_ss, cv_sh;     // row, slot, head
    float *weight;       // DEVICE [batch][n_kv_heads][cap] or null
    int32_t *age;        // DEVICE [batch][n_kv_heads][cap] or null
    int32_t *lens;       // DEVICE [batch]
    unsigned int *ticket;   // DEVICE [batch]: arrivals of a row's insert CTAs, left zero by each call
    int32_t *gone;          // DEVICE [batch], behind ticket: entries that a truncation takes from each row
    // attention of the whole batch over the prompt on the tensor cores (cstr_prefix.cu)
    int has_maps;        // the copy engine can read the prompt: maps and scratch below are there
    alignas(64) unsigned char map_k[128], map_v[128];     // tensor maps of prefix_k, prefix_v
    float *part_o;       // DEVICE parts' outputs, [block][head_dim (padded) / 4][128][4]
    void *part_ml;       // DEVICE float2 [block][128]: parts' maximum and sum
    int *status;         // DEVICE [1]: CTAs whose bounded waits gave up (never expected)
    int32_t *list;       // DEVICE [batch][n_kv_heads][2][cap]: the insert kernel's keys and places, where
                         // they are not in shared memory
};

// n / d for 0 <= n < 2^31 by a multiplication: mul = ceil(2^(31 + log) / d), log = ceil(log2 d),
// n mul / 2^(31 + log) = (high word of 2 n x mul) / 2^log
struct cstr_divisor {
    unsigned mul;
    int log;
    __host__ void set(unsigned d)
    {
        log = 0;
        while ((1ull << log) < d)
            ++log;
        mul = (unsigned)(((1ull << (31 + log)) + d - 1) / d);
    }
    __device__ __forceinline__ int operator()(int n) const
    {
        return (int)(__umulhi(2u * (unsigned)n, mul) >> log);
    }
};

// Attention of the rows' own keys (and of prefix keys not taken by another kernel).
struct cstr_row_args {
    const void *q;
    int64_t q_sb, q_st, q_sh;
    void *out;
    int64_t o_sb, o_st, o_sh;
    float *lse_out;      // [batch][tokens][heads] or null
    int32_t tokens;
    const int32_t *pos, *n_query;
    float scale_log2;    // softmax scale x log2(e)
    int32_t accumulate;
};
// with_prefix: the prompt's keys belong to the row kernel's lists; else cstr_launch_prefix has
// been launched before on the stream, and its parts are joined
int cstr_launch_row_attention(const cstr_cache &c, const cstr_row_args &a, bool with_prefix,
                              cudaStream_t stream);

// How the prefix kernel deals its work out: `pairs` groups of 256 query rows per key / value head,
// `tiles` key tiles of 128; units (head, group, tile) in this order, CTA i of `grid` takes
// [i units / grid, (i + 1) units / grid).
struct cstr_prefix_plan {
    int pairs, tiles, grid;
};
cstr_prefix_plan cstr_plan_prefix(const cstr_cache &c, int tokens);
int cstr_prefix_init(cstr_cache *c);
int cstr_launch_prefix(const cstr_cache &c, const cstr_row_args &a, cudaStream_t stream);

struct cstr_insert_args {
    const void *k_new, *v_new;
    int64_t k_sb, k_st, k_sh, v_sb, v_st, v_sh;
    int32_t tokens;
    const int32_t *n_new, *pos;
    int32_t budget, recent;
    int32_t back;        // no insertion: entries of age pos or more leave
};
int cstr_launch_insert(const cstr_cache &c, const cstr_insert_args &a, cudaStream_t stream);

// Largest cap whose keys and places fit the insert kernel's shared memory (8 bytes a slot beside
// 8 KB of bins).
#define CSTR_INSERT_SMEM_SLOTS 24576
// Largest cap whose single tokens a warp per item inserts; where it has more than one entry to evict
// (a shrinking row), its keys and places are in scratch, too.
#define CSTR_INSERT_WARP_SLOTS 2048
