// Key / value cache of a batch with a shared prompt: handle, argument checks,
// the insertion of new tokens with eviction by accumulated attention weight, and
// the removal of tokens that are taken back.
#include <math.h>
#include <string.h>

#include <new>

#include "cstr_cache.cuh"

namespace {

// ---- insertion -------------------------------------------------------------
//
// Per row and key / value head ("item"), entries are ordered by (protected,
// weight, slot); their 32-bit keys are order-preserving bits of the weight, all
// ones when protected, 0 for NaN.  The e-th smallest key is found, ties at it are
// taken in slot order, evicted slots below the new length and surviving ones past
// it are listed in slot order, and the i-th free place gets the i-th mover.
// All of it is counting, so no result depends on the order of atomics.
//
// Bound: 8 bytes per entry (weight, age) are read; only new tokens, and
// survivors past the new length, are copied.  What costs time beyond that is the
// chain of dependent steps of one item, so the variants differ in who
// works on it:
//   single tokens, up to 2,048 slots: a warp per item.  It evicts one entry (a
//     decoding step with a full cache): the smallest (key, slot) pair, found
//     while the row is read, without a barrier.  512 rows x 8 heads of 1,024 slots
//     10.3 us (33.7 MB, 3.3 TB/s; a CTA per item 27.3 us), of 2,048 17.4 us (33.7);
//     past that the CTA wins: 128 x 8 of 4,096 11.4 us, a warp 16.2 us;
//   else a CTA per item, 256 threads up to 4,096 slots (so that several items share
//     an SM), 1,024 beyond: 64 rows x 8 heads of 2,304 slots, 256 tokens 31.0 us (75 MB,
//     2.4 TB/s; with 1,024 threads 43.8 us), of 8,192 slots 62.4 us (with 256 60.2 us),
//     few rows of more, 4 x 8 of 20,000, 64 tokens 25.8 us (48.5).  Keys in shared memory
//     (or scratch, past 24,576: at 8,192 slots 65.1 us, at 2,304 32.3 us), the e-th
//     smallest from counts per 11-bit digit.
// Tokens that are taken back leave by the same kernel, a CTA per item, with keys that put them first; a
// kernel before it counts them per row (512 rows x 8 heads of 1,024 slots, three tokens: 17 us together).
constexpr int kMaxThreads = 1024;
constexpr int kMaxWarps = kMaxThreads / 32;


struct InsertParams {
    const char *k_new, *v_new;
    long long nk_sb, nk_st, nk_sh, nv_sb, nv_st, nv_sh;
    char *ck, *cv;
    long long ck_sb, ck_ss, ck_sh, cv_sb, cv_ss, cv_sh;
    float *weight;
    int32_t *age, *lens;
    const int32_t *n_new, *pos;
    unsigned int *ticket;
    int32_t *gone;       // tokens taken back: entries that leave each row (null: insertion)
    int32_t *list;       // null: keys and places live in shared memory
    int B, Hk, D, cap, T, budget, recent;
    int bits;            // of a digit: 11 (8 KB of bins) or 8 (1 KB, for CTAs that hardly ever count)
    int wide;            // weight and age rows can be read 16 bytes at a time
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

constexpr unsigned kZeroKey = 0x80000000u;    // evict_key of weight 0

// Tokens taken back: entries of age `from` or more are the first to leave.
__device__ __forceinline__ unsigned back_key(float w, int age, int from)
{
    return age >= from ? 0u : max(evict_key(w, age, INT_MAX), 1u);      // (INT_MAX is `from` or more)
}

// f(slot, key) for the slots [0, len) of a row, each by one of `step` threads; BACK: the keys of back_key, with
// `from` in the place of protect_from
template <bool BACK, typename F>
__device__ __forceinline__ void for_keys(const InsertParams &p, const float *weight, const int32_t *age, int len,
                                         int protect_from, int tid, int step, F f)
{
    auto evict_key = [](float w, int age, int limit) {
        return BACK ? back_key(w, age, limit) : ::evict_key(w, age, limit);
    };
    if (p.wide) {
#pragma unroll 1
        for (int j0 = tid * 4; j0 < len; j0 += step * 16) {       // eight loads in flight
            float4 w[4];
            int4 a[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = j0 + i * step * 4;
                if (j < len) {
                    w[i] = *reinterpret_cast<const float4 *>(weight + j);
                    a[i] = *reinterpret_cast<const int4 *>(age + j);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = j0 + i * step * 4;
                if (j < len)
                    f(j, evict_key(w[i].x, a[i].x, protect_from));
                if (j + 1 < len)
                    f(j + 1, evict_key(w[i].y, a[i].y, protect_from));
                if (j + 2 < len)
                    f(j + 2, evict_key(w[i].z, a[i].z, protect_from));
                if (j + 3 < len)
                    f(j + 3, evict_key(w[i].w, a[i].w, protect_from));
            }
        }
    } else {
#pragma unroll 4
        for (int j = tid; j < len; j += step)
            f(j, evict_key(weight[j], age[j], protect_from));
    }
}

template <bool WARP> __device__ __forceinline__ void team_sync()
{
    if (WARP)
        __syncwarp();
    else
        __syncthreads();
}

// Evicted: key < limit, and the first `want` slots with key == limit (`all_equal`: all of them, so that
// they need no counting).  Lists the free places below
// new_len (ascending, from place[0]) and the surviving slots at or past it (ascending, from
// place[cap - 1] downwards); returns the number of the latter.  The team is a warp or the CTA; its
// warps own contiguous spans [lo, hi) of slots.
template <bool WARP>
__device__ __forceinline__ int list_places(const InsertParams &p, const unsigned *keys, int *place, int *s_word, int len, int new_len,
                                           unsigned limit, int want, bool all_equal, int lo, int hi)
{
    const int lane = threadIdx.x & 31, warp = WARP ? 0 : threadIdx.x >> 5;
    const int warps = WARP ? 1 : blockDim.x >> 5, tid = WARP ? lane : threadIdx.x, step = WARP ? 32 : blockDim.x;
    const unsigned below = (1u << lane) - 1u;
    int tie0 = 0;
    if (!all_equal) {
        int ties = 0;
#pragma unroll 4
        for (int j = lo + lane; j - lane < hi; j += 32)
            ties += __popc(__ballot_sync(0xffffffffu, j < hi && keys[j] == limit));
        if (lane == 0)
            s_word[warp] = ties;
        team_sync<WARP>();
        if (!WARP)
            tie0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_word[lane] : 0);
        team_sync<WARP>();
    }
    int holes = 0, movers = 0;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {                     // count, then write
        int hole0 = 0, mover0 = 0, tie = tie0;
        if (round == 1) {
            if (lane == 0)
                s_word[warp] = holes, s_word[kMaxWarps + warp] = movers;
            team_sync<WARP>();
            if (!WARP) {
                hole0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_word[lane] : 0);
                mover0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_word[kMaxWarps + lane] : 0);
            }
        }
        holes = movers = 0;
#pragma unroll 4
        for (int j = lo + lane; j - lane < hi; j += 32) {
            const unsigned k = j < hi ? keys[j] : 0xffffffffu;
            const unsigned equal = __ballot_sync(0xffffffffu, j < hi && k == limit);
            const bool gone = j < hi && (k < limit || (k == limit && (all_equal || tie + __popc(equal & below) < want)));
            tie += __popc(equal);
            const unsigned hole = __ballot_sync(0xffffffffu, gone && j < new_len);
            const unsigned mover = __ballot_sync(0xffffffffu, j < hi && !gone && j >= new_len);
            if (round == 1) {
                if (gone && j < new_len)
                    place[hole0 + holes + __popc(hole & below)] = j;
                if (j < hi && !gone && j >= new_len)
                    place[p.cap - 1 - (mover0 + movers + __popc(mover & below))] = j;
            }
            holes += __popc(hole);
            movers += __popc(mover);
        }
        if (round == 1 && warp == warps - 1 && lane == 0) {       // totals
            s_word[2 * kMaxWarps] = hole0 + holes;
            s_word[2 * kMaxWarps + 1] = mover0 + movers;
        }
    }
    team_sync<WARP>();
    const int all = s_word[2 * kMaxWarps];
    for (int j = len + tid; j < new_len; j += step)               // free places past the old length
        place[all + j - len] = j;
    team_sync<WARP>();
    return s_word[2 * kMaxWarps + 1];
}

// Reads a row, leaves its keys in keys[0 .. len), and finds the `evict` smallest: those below the
// returned limit and the first `want` (in slot order) of the `equal` ones at it; where all of these
// belong to them, the limit may be any larger key below the next one.  Counts per digit of p.bits
// bits, the most significant first (that one while the row is read).
template <bool WARP, bool BACK>
__device__ __forceinline__ unsigned select_by_digits(const InsertParams &p, const float *weight, const int32_t *age,
                                                     int protect_from, unsigned *keys, int *s_bin, int *s_word,
                                                     int len, int evict, int &want, int &equal)
{
    const int lane = threadIdx.x & 31, warp = WARP ? 0 : threadIdx.x >> 5;
    const int tid = WARP ? lane : threadIdx.x, step = WARP ? 32 : blockDim.x;
    const int per = (1 << p.bits) / step;                         // bins of a thread, side by side
    int *mine = s_bin + tid * per;
    unsigned prefix = 0, fixed = 0;                               // digits found so far, and their mask
    want = evict;                                                 // rank among the keys with this prefix
    auto clear = [&] {                                            // (per is 2, 8 or 64; bins are aligned)
        if (per % 4 == 0)
            for (int i = 0; i < per; i += 4)
                *reinterpret_cast<int4 *>(mine + i) = make_int4(0, 0, 0, 0);
        else
            for (int i = 0; i < per; ++i)
                mine[i] = 0;
    };
    clear();
    team_sync<WARP>();
#pragma unroll 1
    for (int left = 32; left > 0; left -= p.bits) {
        const int shift = max(left - p.bits, 0);
        const unsigned digits = (1u << (left - shift)) - 1u;
        // Protected entries, and tokens that nothing has attended to yet, are many: they would queue up
        // at one bin.  The former are left out, the latter are counted aside.
        int zeros = 0;
        auto count = [&](unsigned k) {
            if (k == kZeroKey)
                ++zeros;
            else if (k != 0xffffffffu)
                atomicAdd(&s_bin[(k >> shift) & digits], 1);
        };
        if (left == 32) {
            for_keys<BACK>(p, weight, age, len, protect_from, tid, step, [&](int j, unsigned k) {
                keys[j] = k;
                count(k);
            });
        } else {
#pragma unroll 4
            for (int j = tid; j < len; j += step) {
                const unsigned k = keys[j];
                if ((k & fixed) == prefix)
                    count(k);
            }
        }
        __syncwarp();
        zeros = __reduce_add_sync(0xffffffffu, zeros);
        if (lane == 0 && zeros)
            atomicAdd(&s_bin[(kZeroKey >> shift) & digits], zeros);
        team_sync<WARP>();
        // first digit whose running count reaches `want`: a thread adds up its bins, the warps scan
        int sum = 0;
        if (per % 4 == 0)
            for (int i = 0; i < per; i += 4) {
                const int4 c = *reinterpret_cast<const int4 *>(mine + i);
                sum += c.x + c.y + c.z + c.w;
            }
        else
            for (int i = 0; i < per; ++i)
                sum += mine[i];
        int upto = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, off);
            upto += lane >= off ? o : 0;
        }
        if (!WARP) {
            if (lane == 31)
                s_word[warp] = upto;
            __syncthreads();
            upto += __reduce_add_sync(0xffffffffu, lane < warp ? s_word[lane] : 0);
        }
        if (upto >= want && upto - sum < want) {                  // one thread, if any
            int before = upto - sum, i = 0;
            while (before + mine[i] < want)
                before += mine[i++];
            s_word[kMaxWarps] = tid * per + i;
            s_word[kMaxWarps + 1] = before;
            s_word[kMaxWarps + 2] = mine[i];
        }
        if (tid == step - 1 && upto < want)                       // protected entries have to go, too
            s_word[kMaxWarps] = -1, s_word[kMaxWarps + 1] = upto;
        clear();                                                  // for the next digit
        team_sync<WARP>();
        const int d = s_word[kMaxWarps];
        want -= s_word[kMaxWarps + 1];
        if (d < 0) {
            prefix = 0xffffffffu;
            equal = -1;
            break;
        }
        prefix |= (unsigned)d << shift;
        fixed |= digits << shift;
        equal = s_word[kMaxWarps + 2];
        if (equal == want) {                                      // no need to tell these apart
            prefix |= ~fixed;
            break;
        }
    }
    team_sync<WARP>();
    return prefix;
}

// BACK: no new tokens; p.gone[row] entries leave, those of age p.pos[row] or more first
template <bool WARP, bool BACK>
__global__ void __launch_bounds__(WARP ? 128 : kMaxThreads, WARP ? 8 : 1)
cache_insert_kernel(const __grid_constant__ InsertParams p)
{
    constexpr int kWords = 2 * kMaxWarps + 2;
    extern __shared__ __align__(16) int s_dyn[];                  // bins, keys, places
    __shared__ int s_words[(WARP ? 4 : 1) * kWords];
    __shared__ unsigned long long s_least[kMaxWarps];
    cstr_wait_for_earlier_kernels();
    cstr_let_next_kernel_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tid = WARP ? lane : threadIdx.x, step = WARP ? 32 : blockDim.x;
    const int item = WARP ? blockIdx.x * 4 + warp : blockIdx.x;
    if (item >= p.B * p.Hk)
        return;                                                   // (a whole warp; no CTA barrier follows)
    const int b = item / p.Hk, kh = item - b * p.Hk;
    const int len = min(max(p.lens[b], 0), p.cap);
    const int n = BACK ? 0 : p.n_new ? min(max(p.n_new[b], 0), p.T) : p.T;
    const int pos = p.pos[b];
    const int new_len = BACK ? len - p.gone[b] : min(len + n, p.budget);
    const int evict = len + n - new_len;
    const int protect_from = BACK ? pos : pos + n - p.recent;
    const long long entry0 = (long long)item * p.cap;
    float *weight = p.weight + entry0;
    int32_t *age = p.age + entry0;
    int *s_bin = s_dyn + (WARP ? warp << p.bits : 0), *s_word = s_words + (WARP ? warp * kWords : 0);
    unsigned *keys = reinterpret_cast<unsigned *>(p.list ? p.list + entry0 * 2 : s_dyn + (1 << p.bits));
    int *place = reinterpret_cast<int *>(keys + p.cap);
    int n_old = 0;                                                // survivors past the new length
    int only = len;                                               // evict == 1: the evicted slot
    const bool listed = evict > 1;

    if (listed) {
        if (!WARP) {                                              // the new tokens are on their way meanwhile
            const int lines = (p.D * 2 + 127) / 128;
            for (int i = tid; i < n * lines; i += step) {
                const int t = i / lines, line = i - t * lines;
                const char *k = p.k_new + ((long long)b * p.nk_sb + (long long)t * p.nk_st + (long long)kh * p.nk_sh) * 2;
                const char *v = p.v_new + ((long long)b * p.nv_sb + (long long)t * p.nv_st + (long long)kh * p.nv_sh) * 2;
                asm volatile("prefetch.global.L2 [%0];" ::"l"(k + line * 128));
                asm volatile("prefetch.global.L2 [%0];" ::"l"(v + line * 128));
            }
        }
        int want, equal;
        const unsigned limit = select_by_digits<WARP, BACK>(p, weight, age, protect_from, keys, s_bin, s_word, len, evict,
                                                      want, equal);
        const int warps = WARP ? 1 : blockDim.x >> 5, span = ((len + warps - 1) / warps + 31) & ~31;
        const int lo = WARP ? 0 : min(warp * span, len), hi = min(lo + span, len);
        n_old = list_places<WARP>(p, keys, place, s_word, len, new_len, limit, want, equal == want, lo, hi);
    } else if (evict == 1) {
        unsigned long long least = ~0ull;
        for_keys<BACK>(p, weight, age, len, protect_from, tid, step, [&](int j, unsigned k) {
            const unsigned long long at = ((unsigned long long)k << 32) | (unsigned)j;
            least = at < least ? at : least;
        });
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const unsigned long long o = __shfl_xor_sync(0xffffffffu, least, off);
            least = o < least ? o : least;
        }
        if (!WARP) {
            if (lane == 0)
                s_least[warp] = least;
            __syncthreads();
            for (int w = 0; w < (int)(blockDim.x >> 5); ++w)
                least = s_least[w] < least ? s_least[w] : least;
        }
        only = (int)(unsigned)least;
        // with nothing added the last entry lies past the new length, and fills the evicted slot
        // unless it is the evicted one itself
        n_old = n == 0 && only < new_len ? 1 : 0;
    }
    // free places: the list; or the evicted slot and then [len, new_len); or [len, new_len)
    const int moves = n_old + n;
    auto place_of = [&](int mv) {
        if (listed)
            return place[mv];
        return evict == 1 ? (mv == 0 ? only : len + mv - 1) : len + mv;
    };
    auto mover = [&](int mv) { return listed ? place[p.cap - 1 - mv] : len - 1; };

    // copies: 16 bytes a thread, keys and values of four places in flight
    const int per = p.D / 8, at_once = step / per;                // pieces of a row; places side by side
    const int piece = tid % per;
    char *ck = p.ck + ((long long)b * p.ck_sb + (long long)kh * p.ck_sh) * 2 + piece * 16;
    char *cv = p.cv + ((long long)b * p.cv_sb + (long long)kh * p.cv_sh) * 2 + piece * 16;
    const char *nk = p.k_new + ((long long)b * p.nk_sb + (long long)kh * p.nk_sh) * 2 + piece * 16;
    const char *nv = p.v_new + ((long long)b * p.nv_sb + (long long)kh * p.nv_sh) * 2 + piece * 16;
    if (tid < at_once * per) {
        for (int mv0 = tid / per; mv0 < moves; mv0 += 4 * at_once) {
            uint4 k[4], v[4];
            int dst[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int mv = mv0 + i * at_once;
                dst[i] = -1;
                if (mv >= moves)
                    continue;
                const bool old = mv < n_old;
                const int from = old ? mover(mv) : mv - n_old;
                dst[i] = place_of(mv);
                if (!CSTR_INB(p.oob, dst[i], p.cap, CSTR_SITE_CACHE) ||
                    !CSTR_INB(p.oob, from, old ? p.cap : p.T, CSTR_SITE_CACHE)) {
                    dst[i] = -1;
                    continue;
                }
                k[i] = *reinterpret_cast<const uint4 *>(old ? ck + from * p.ck_ss * 2 : nk + from * p.nk_st * 2);
                v[i] = *reinterpret_cast<const uint4 *>(old ? cv + from * p.cv_ss * 2 : nv + from * p.nv_st * 2);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (dst[i] < 0)
                    continue;
                *reinterpret_cast<uint4 *>(ck + dst[i] * p.ck_ss * 2) = k[i];
                *reinterpret_cast<uint4 *>(cv + dst[i] * p.cv_ss * 2) = v[i];
            }
        }
    }
    for (int mv = tid; mv < moves; mv += step) {
        const int dst = place_of(mv);
        if (!CSTR_INB(p.oob, dst, p.cap, CSTR_SITE_CACHE))
            continue;
        if (mv < n_old) {
            const int j = mover(mv);
            weight[dst] = weight[j];
            age[dst] = age[j];
        } else {
            weight[dst] = 0.f;
            age[dst] = pos + mv - n_old;
        }
    }

    // every team of the row has read lens[b] when it arrives here; the last one replaces it
    team_sync<WARP>();
    if (tid == 0) {
        const unsigned prev = atomicAdd(p.ticket + b, 1u);
        if (prev == (unsigned)p.Hk - 1u) {
            p.ticket[b] = 0u;
            p.lens[b] = new_len;
        }
    }
}

// gone[row] = entries of age pos[row] or more in the head that has the most of them; a block per row
__global__ void __launch_bounds__(256)
cache_count_kernel(const __grid_constant__ InsertParams p)
{
    __shared__ int s_most[8];
    cstr_wait_for_earlier_kernels();
    cstr_let_next_kernel_start();
    const int b = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int len = min(max(p.lens[b], 0), p.cap), pos = p.pos[b];
    int most = 0;
    for (int kh = warp; kh < p.Hk; kh += 8) {
        const int32_t *age = p.age + ((long long)b * p.Hk + kh) * p.cap;
        int n = 0;
#pragma unroll 8
        for (int j = lane; j < len; j += 32)
            n += age[j] >= pos;
        most = max(most, __reduce_add_sync(0xffffffffu, n));
    }
    if (lane == 0)
        s_most[warp] = most;
    __syncthreads();
    if (warp == 0) {
        most = __reduce_max_sync(0xffffffffu, lane < 8 ? s_most[lane] : 0);
        if (lane == 0)
            p.gone[b] = most;
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

namespace {

// a block per item
template <bool BACK>
int launch_blocks(const cstr_cache &c, InsertParams &p, unsigned items, cudaStream_t stream)
{
    const bool shared = c.cap <= CSTR_INSERT_SMEM_SLOTS;
    if (shared)
        p.list = nullptr;
    p.bits = 11;
    const int smem = (4 << p.bits) + (shared ? c.cap * 8 : 0);
    static std::atomic<bool> allowed[64];
    const int rc = cstr_allow_smem(cache_insert_kernel<false, BACK>, allowed, c.device,
                                   (4 << p.bits) + CSTR_INSERT_SMEM_SLOTS * 8);
    if (rc)
        return rc;
    return cstr_launch(cache_insert_kernel<false, BACK>, items, c.cap <= 4096 ? 256 : kMaxThreads, 1, smem, stream, p);
}

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
    p.wide = c.cap % 4 == 0 && aligned16(c.weight) && aligned16(c.age);
    const unsigned items = (unsigned)(c.batch * c.n_kv_heads);
    if (a.back) {
        p.gone = c.gone;
        const int rc = cstr_launch(cache_count_kernel, c.batch, 256, 1, 0, stream, p);
        return rc ? rc : launch_blocks<true>(c, p, items, stream);
    }
    if (a.tokens == 1 && c.cap <= CSTR_INSERT_WARP_SLOTS) {
        p.bits = 8;
        return cstr_launch(cache_insert_kernel<true, false>, (items + 3) / 4, 128, 1, 4 * (4 << p.bits), stream, p);
    }
    return launch_blocks<false>(c, p, items, stream);
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
        e = cudaMalloc((void **)&c->ticket, (size_t)batch * 8);
    c->gone = (int32_t *)(c->ticket + batch);
    if (e == cudaSuccess)
        e = cudaMalloc((void **)&c->status, 4);
    if (e == cudaSuccess && weight && age && (cap <= CSTR_INSERT_WARP_SLOTS || cap > CSTR_INSERT_SMEM_SLOTS))
        e = cudaMalloc((void **)&c->list, (size_t)batch * n_kv_heads * cap * 8);
    // zeroed before the handle is out, whatever stream it is used on and whatever the default stream has queued
    cudaStream_t own = nullptr;
    if (e == cudaSuccess)
        e = cudaStreamCreateWithFlags(&own, cudaStreamNonBlocking);
    if (e == cudaSuccess)
        e = cudaMemsetAsync(c->ticket, 0, (size_t)batch * 4, own);
    if (e == cudaSuccess)
        e = cudaMemsetAsync(c->status, 0, 4, own);
    if (e == cudaSuccess)
        e = cudaStreamSynchronize(own);
    if (own)
        cudaStreamDestroy(own);
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

extern "C" int cstr_cache_truncate(cstr_cache_t *c, const int32_t *pos, void *cuda_stream)
{
    if (!c || !pos)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_truncate: null pointer");
    if (!c->weight || !c->age)
        return cstr_fail(CSTR_ERR_NULL, "cstr_cache_truncate: the cache was created without weight or age");
    const int rc = cstr_check_device(c->device, "cache");
    if (rc)
        return rc;
    cstr_insert_args a;
    memset(&a, 0, sizeof a);
    a.pos = pos;
    a.back = 1;
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
    const float scale_log2 = (float)((double)scale * 1.4426950408889634);
    if (!isfinite(scale_log2))
        return cstr_fail(CSTR_ERR_ARG, "cstr_cache_attention: scale x log2(e) = %g is not finite", scale_log2);
    int rc = strides_ok("cstr_cache_attention", q_strides, 3);
    if (!rc)
        rc = strides_ok("cstr_cache_attention", out_strides, 3);
    if (rc)
        return rc;
    for (int i = 0; i < 3; ++i)
        if (q_strides[i] > (1ll << 33) || q_strides[i] < -(1ll << 33))
            return cstr_fail(CSTR_ERR_SHAPE, "cstr_cache_attention: q stride %lld is too large", (long long)q_strides[i]);
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
    a.scale_log2 = scale_log2;
    a.accumulate = accumulate ? 1 : 0;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    // On the tensor cores the prompt costs a launch and the join of its parts, about 10 us; in the row kernel
    // every row reads it by itself, from the L2 cache mostly, and few rows in a long serial chain each.
    // So: from 512 tokens on, or where the rows read 16 MiB of it together, 32 MiB if they have no more than 8
    // query rows for it.  Measured in us, tensor / row, head_dim 128:
    //   8 query rows, 8 key / value heads: 4 x 512 tokens 12.2 / 12.9, 1 x 1,024 12.9 / 13.7, 64 x 256 17.3 / 22.5
    //   (64 MiB); 2 heads: 64 x 256 (16 MiB) 16.6 / 12.7, 128 x 256 (32 MiB) 16.8 / 15.9, 256 x 256 17.3 / 22.5,
    //   64 x 512 16.8 / 16.1, 64 x 1,024 17.2 / 22.7; 1 head: 128 x 384 (24 MiB) 21.3 / 13.6
    //   16 query rows, 16 MiB: 128 x 1 head x 256 18.0 / 23.2, 16 x 8 x 256 18.2 / 23.6
    // What the rule misses: one row of 16 to 32 query rows, 512 to 4,096 tokens (1 x 4,096 26.2 / 23.1, 39.0 / 32.9).
    const long long reads = (long long)c->batch * c->n_kv_heads * c->prefix_len * c->head_dim * 4;
    const bool narrow = (long long)n_tokens * (c->n_heads / c->n_kv_heads) <= 8;
    const bool tensor = c->has_maps && c->prefix_len >= 128 &&
                        (c->prefix_len >= 512 || reads >= (narrow ? 32 << 20 : 16 << 20));
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
