// Rows of logits under their automaton states, as the operators on whole distributions read them:
// the tables' descriptors and their host checks, a row's mask, masked vectors of logits, the next
// state, and exponentials in 64 bits.
#pragma once

#include <math_constants.h>

#include <atomic>

#include "cstr_internal.cuh"

namespace cstr_rows {

constexpr unsigned kFull = 0xffffffffu;

struct TableDesc {
    const uint32_t *mask;
    const void *next;        // token-major: next[token * lds + internal state]
    const uint8_t *accept;
    const int32_t *rank;     // caller's state id -> internal one, or null (identity)
    const int32_t *unrank;   // and back
    long long lds, ldw;
    int n_states, wide, code_shift;
};

struct Tables {
    TableDesc tab[CSTR_MAX_TABLES];
    int n;                   // 0: every token is allowed
    const int32_t *row_table, *states;
};

// Checks of the arguments that the row operators share; fills `out`.
inline int take_tables(const char *name, const cstr_table_t *const *tables, int32_t n_tables, const int32_t *row_table,
                       const int32_t *states, int32_t vocab_size, int device, Tables &out)
{
    out.n = n_tables;
    out.row_table = row_table;
    out.states = states;
    for (int32_t i = 0; i < n_tables; ++i) {
        const cstr_table *t = tables[i];
        if (!t)
            return cstr_fail(CSTR_ERR_NULL, "%s: tables[%d] is null", name, i);
        if (t->device != device)
            return cstr_fail(CSTR_ERR_DEVICE, "%s: tables[%d] is on device %d, device %d is current", name, i,
                             t->device, device);
        if (t->n_states < 1)
            return cstr_fail(CSTR_ERR_ARG, "%s: tables[%d] has not been built", name, i);
        if (t->V != vocab_size)
            return cstr_fail(CSTR_ERR_SHAPE, "%s: tables[%d] has V = %d, vocab_size is %d", name, i, t->V, vocab_size);
        TableDesc &d = out.tab[i];
        d.mask = t->mask;
        d.next = t->next;
        d.accept = t->accept;
        d.rank = t->renumbered ? t->rank : nullptr;
        d.unrank = t->renumbered ? t->unrank : nullptr;
        d.lds = t->lds;
        d.ldw = t->ldw;
        d.n_states = t->n_states;
        d.wide = t->wide;
        d.code_shift = t->code_shift;
    }
    return CSTR_OK;
}

// Limits of a kernel that its launches may need, set once per device, always to the same values: calls from several
// threads may not undo each other's.
template <int kKinds> struct LaunchLimits {
    std::atomic<bool> done[64][kKinds];
    template <class K> int set(K kernel, int kind, int device, int cluster, int smem)
    {
        if (device >= 0 && device < 64 && done[device][kind].load(std::memory_order_acquire))
            return CSTR_OK;
        if (cluster > 8)
            CSTR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        if (smem > 48 * 1024)
            CSTR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (device >= 0 && device < 64)
            done[device][kind].store(true, std::memory_order_release);
        return CSTR_OK;
    }
};

// SMs of a device, asked for once.
inline int sm_count(int device, int &sms)
{
    static std::atomic<int> known[64];
    sms = device >= 0 && device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
    if (sms > 0)
        return CSTR_OK;
    CSTR_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    if (device >= 0 && device < 64)
        known[device].store(sms, std::memory_order_relaxed);
    return CSTR_OK;
}

// The row's table and state; false: an inactive row.  mrow: its mask, null where everything is allowed.
__device__ __forceinline__ bool row_state(const Tables &a, int row, int &table, int &state, const uint32_t *&mrow)
{
    mrow = nullptr;
    table = 0;
    state = -1;
    if (a.n == 0)
        return true;
    table = a.row_table ? a.row_table[row] : 0;
    state = a.states[row];
    if (table < 0 || table >= a.n || state < 0 || state >= a.tab[table].n_states)
        return false;
    mrow = a.tab[table].mask + (long long)state * a.tab[table].ldw;
    return true;
}

// State after an allowed token from internal state `inner` (next holds codes of internal ids; its sink means
// "no edge").
__device__ __forceinline__ int next_state(const TableDesc &t, int inner, int token)
{
    const long long at = (long long)token * t.lds + inner;
    int q = t.wide ? ((const int32_t *)t.next)[at] : (int)((const uint16_t *)t.next)[at];
    q = CSTR_UNPERM(q >> t.code_shift);
    return q == t.n_states ? CSTR_DEAD : t.unrank ? t.unrank[q] : q;
}

// A row as 16-byte vectors from the 16-byte boundary at or before its first logit: vector v holds the
// tokens v * N - head .. + N - 1, those outside [0, V) read as disallowed and not touched.
template <bool BF16> struct RowView {
    static constexpr int N = BF16 ? 8 : 4, ESZ = BF16 ? 2 : 4;
    const char *row;         // first logit
    const uint32_t *mrow;    // allowed tokens, or null
    int head, V;

    __device__ __forceinline__ RowView(const void *logits, long long offset, int V_, const uint32_t *m)
        : row((const char *)logits + offset * ESZ), mrow(m), V(V_)
    {
        head = (int)((unsigned)(uintptr_t)row & 15u) / ESZ;
    }
    __device__ __forceinline__ int vectors() const { return (V + head + N - 1) / N; }
    __device__ __forceinline__ int token(int v) const { return v * N - head; }
    __device__ __forceinline__ bool inside(int v) const { return token(v) >= 0 && token(v) + N <= V; }
    __device__ __forceinline__ bool allowed(int tok) const { return !mrow || ((__ldg(mrow + (tok >> 5)) >> (tok & 31)) & 1u); }
    __device__ __forceinline__ float one(int tok) const
    {
        return BF16 ? __uint_as_float((unsigned)((const unsigned short *)row)[tok] << 16) : ((const float *)row)[tok];
    }
    // allowed bits of a vector that is inside
    __device__ __forceinline__ unsigned bits(int v) const
    {
        if (!mrow)
            return kFull;
        const int tok = token(v);
        const unsigned lo = __ldg(mrow + (tok >> 5));
        return __funnelshift_r(lo, (tok & 31) + N > 32 ? __ldg(mrow + (tok >> 5) + 1) : 0u, tok & 31);
    }
    // raw vector with -infinity where the token is disallowed
    static __device__ __forceinline__ uint4 mask(uint4 u, unsigned bits)
    {
        unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (BF16)
                w[i] = __byte_perm((bits >> (2 * i)) & 1u ? w[i] : 0xff80ff80u, (bits >> (2 * i + 1)) & 1u ? w[i] : 0xff80ff80u, 0x7610);
            else
                w[i] = (bits >> i) & 1u ? w[i] : 0xff800000u;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // A vector that is partly (or not) inside.  (A loop: it is rare, and its code is in many places.)
    __device__ __forceinline__ uint4 edge(int v) const
    {
        unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll 1
        for (int e = N - 1; e >= 0; --e) {               // into the highest place, moved down by those before it
            const int tok = token(v) + e;
            const unsigned f = __float_as_uint(tok >= 0 && tok < V && allowed(tok) ? one(tok) : -CUDART_INF_F);
            if (BF16) {
                w[3] = w[3] << 16 | w[2] >> 16;
                w[2] = w[2] << 16 | w[1] >> 16;
                w[1] = w[1] << 16 | w[0] >> 16;
                w[0] = w[0] << 16 | f >> 16;
            } else {
                w[3] = w[2];
                w[2] = w[1];
                w[1] = w[0];
                w[0] = f;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ uint4 masked(int v) const
    {
        return inside(v) ? mask(reinterpret_cast<const uint4 *>(row - head * ESZ)[v], bits(v)) : edge(v);
    }
    // Logit e of a raw vector; by value() NaN reads as -infinity.
    static __device__ __forceinline__ float plain(uint4 u, int e)
    {
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
        return BF16 ? __uint_as_float(e & 1 ? w[e / 2 % 4] & 0xffff0000u : w[e / 2 % 4] << 16) : __uint_as_float(w[e % 4]);
    }
    static __device__ __forceinline__ float at(uint4 u, int e)       // ... e known only when it runs
    {
        const int i = BF16 ? e >> 1 : e;
        const unsigned w = i & 2 ? (i & 1 ? u.w : u.z) : (i & 1 ? u.y : u.x);
        return __uint_as_float(!BF16 ? w : e & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ float value(uint4 u, int e) { return fmaxf(plain(u, e), -CUDART_INF_F); }
};

// 2^(d c16 / 16) for d c16 / 16 in [-1020, 0] to 2.6e-12 as a product of the two numbers that it returns:
// d c16 = 16 n + j + g, the polynomial of degree 4 that meets 2^(g / 16) at the five Chebyshev points of
// [-1/2, 1/2] (2.5e-12 at most, exact at 0), and table[j] = 2^(j / 16) with n added to its exponent.  The table's
// 16 numbers fill the 32 banks of shared memory once: lanes never conflict.
__device__ __forceinline__ double2 exp2_factors(double d, double c16, const double *table)
{
    const double shift = 6755399441055744.0;                 // 1.5 * 2^52: adding it rounds to a whole number
    const double r = fma(d, c16, shift), g = fma(d, c16, shift - r);
    double p = 1.467638723829912e-07;
    p = fma(p, g, 1.3551205154934813e-05);
    p = fma(p, g, 0.0009383847926296651);
    p = fma(p, g, 0.043321698760160544);
    p = fma(p, g, 1.0);
    const int i = __double2loint(r);
    const double t = table[i & 15];
    return make_double2(p, __hiloint2double(__double2hiint(t) + ((i >> 4) << 20), __double2loint(t)));
}
// 2^(d c16 / 16) for any d c16 <= 0
__device__ __forceinline__ double exp2_64(double d, double c16, const double *table)
{
    if (!(d * c16 > -16000.0))
        return 0.0;
    const double2 f = exp2_factors(d, c16, table);
    return f.x * f.y;
}

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

}  // namespace cstr_rows
