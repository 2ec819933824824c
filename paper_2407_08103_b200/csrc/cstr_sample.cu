// Sampling under the constraint with temperature, top-k, top-p and min-p from one uniform number a
// row, and the most likely allowed tokens with their log probabilities, each in one kernel.
//
// Mathematics.  The allowed tokens of a row are ordered by (logit descending, id ascending); each of the
// three cuts keeps a prefix of that order, so all of them together keep "logit > x, or logit = x and id <= i"
// for one pair (x, i).  With weights w_v = 2^(c (x_v - m)), c = log2(e) / temperature, m the row's maximum, the
// token is the first one by id whose running sum over the kept weights exceeds u times their sum.  Borders
// between tokens lie 1 / V apart, so that sums in 32 bits would take a neighbour now and then: the weights that
// decide are taken in double precision, to 2.6e-12 of themselves, and weights of single tokens are added as whole
// numbers of 2^-s (s = 62 - log2 V), whose sums are exact whatever their order, atomics included.  Chunks of a row
// that count as a whole (without a cut, with top_p alone, above the border of a wide nucleus) are summed in double
// precision and rounded to such a number once: where a chunk begins depends on the rows of the launch, and its last
// units of 2^-s with it.
//
// A cluster of up to 16 CTAs shares a row.  One pass over memory (the bound: 512 x 256,000 fp32 84 of 116 us, 6.2 of
// 6.55 TB/s in it) leaves the maximum of every lane's logits, and maxima and sums of chunks.  The k-th largest of the
// lanes' maxima is a lower bound of the k-th largest logit, and the mass that they hold one of the row's: so a
// histogram of them tells which few lanes hold every token that can be kept, and only those are looked at again.
// The candidates meet in a list of the first CTA, where they are compared with each other.  Where too many tokens
// can be kept (a nucleus of thousands, many equal logits) the row is read again from the L2 cache: two histograms
// by weights in 32 bits bring the border down to some hundred tokens, one pass counts what lies above them and puts
// them into the list (300 x 128,256 with top_p 0.95, a quarter of the rows that wide, 226 - 268 us by the rows' widths; by
// three exact histograms with 64-bit counters 998 us).  Without any cut the weights of all tokens are needed in 64 bits in the
// first pass; that is bound by the double precision pipe (512 x 256,000 150 us of it).
#include <cooperative_groups.h>
#include <float.h>
#include <math.h>
#include <string.h>

#include "cstr_rows.cuh"

namespace cg = cooperative_groups;

namespace {

using namespace cstr_rows;
typedef unsigned long long u64;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;
constexpr int kU = 4;                     // vectors of a lane in flight: a block is 32 * kU vectors
constexpr int kMaxChunks = 128;           // chunks of a CTA, each of some blocks
constexpr int kDigit = 9, kBins = 1 << kDigit;   // digits of a selection round, distances from the maximum
constexpr int kList = 2048;               // entries of the list, and of the work space behind it
constexpr int kNone = 0x7fffffff;

struct SampleParams {
    Tables t;
    const void *logits;
    long long ld;
    int V, rows;
    int per, blocks;                      // chunks of a CTA, at most; blocks of a chunk
    int scale_bits;                       // s
    u64 *oob;
    // sampling
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *states_out, *tokens;
    float *logp, *kept;
    uint8_t *accept_out;
    // most likely tokens
    int n;
    double c;                             // log2(e) / temperature
    int32_t *ids;
    float *lse;
};

// Ascending for descending logits; -0 and +0 are one value.
__device__ __forceinline__ unsigned order_of(float x)
{
    const unsigned u = __float_as_uint(x + 0.0f);
    return (u & 0x80000000u) ? u : ~(u | 0x80000000u);
}
__device__ __forceinline__ float logit_of(unsigned o)
{
    return __uint_as_float((o & 0x80000000u) ? o : ~o & 0x7fffffffu);
}

// The whole number at or above (below) a * f, for 0 <= f < 1: f is a whole number of 2^-150.
__device__ __forceinline__ u64 part_of(u64 a, float f, bool up)
{
    const unsigned b = __float_as_uint(f);
    const int e = (int)(b >> 23);
    const u64 mant = (b & 0x7fffffu) | (e ? 0x800000u : 0u);
    const int shift = 150 - (e ? e : 1);                     // f = mant * 2^-shift, shift >= 24
    const u64 lo = a * mant, hi = __umul64hi(a, mant);
    if (shift >= 128)
        return up && (lo | hi) ? 1 : 0;
    u64 whole, rest;
    if (shift >= 64) {
        whole = shift == 64 ? hi : hi >> (shift - 64);
        rest = lo | (shift == 64 ? 0 : hi << (128 - shift));
    } else {
        whole = (lo >> shift) | (hi << (64 - shift));
        rest = lo << (64 - shift);
    }
    return whole + (up && rest ? 1 : 0);
}

// s += 2^(c (x - ref)) for two logits, two to an instruction but for the exponential itself
__device__ __forceinline__ void add_exponentials(float2 &s, float x, float y, float ref, float c)
{
    asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %2};\nadd.rn.f32x2 a, a, b;\n"
        "mov.b64 b, {%3, %3};\nmul.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}\n"
        : "+f"(x), "+f"(y) : "f"(-ref), "f"(c));
    x = exp2_fast(x);
    y = exp2_fast(y);
    asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %3};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}\n"
        : "+f"(s.x), "+f"(s.y) : "f"(x), "f"(y));
}

__device__ __forceinline__ u64 inclusive_scan(u64 v, int lane)
{
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const u64 o = __shfl_up_sync(kFull, v, off);
        v += lane >= off ? o : 0;
    }
    return v;
}
__device__ __forceinline__ u64 warp_sum(u64 v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        v += __shfl_xor_sync(kFull, v, off);
    return v;
}
__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        v += __shfl_xor_sync(kFull, v, off);
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        v = fmaxf(v, __shfl_xor_sync(kFull, v, off));
    return v;
}

// What the CTAs of a cluster tell each other.
struct Word {
    double sum;
    u64 mass;
    float m;
    int token;
};

// A prefix of the row's order: logits above x, and those equal to x with ids up to `last`.
struct Cut {
    float x;
    int last;
    __device__ __forceinline__ bool keeps(float v, int tok) const { return v > x || (v == x && tok <= last); }
    __device__ __forceinline__ bool tighter_than(const Cut &o) const { return x > o.x || (x == o.x && last < o.last); }
};

// Bitonic sort of `found` numbers in shared memory (room for the next power of two).
__device__ __forceinline__ void sort_list(u64 *list, int found)
{
    int n = 1;
    while (n < found)
        n <<= 1;
    for (int i = found + threadIdx.x; i < n; i += kThreads)
        list[i] = ~0ull;
    for (int k = 2; k <= n; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < n / 2; i += kThreads) {
                const int a = 2 * i - (i & (j - 1)), b = a + j;
                const u64 x = list[a], y = list[b];
                if ((x > y) == ((a & k) == 0)) {
                    list[a] = y;
                    list[b] = x;
                }
            }
        }
    __syncthreads();
}

template <bool BF16> struct Row {
    using View = RowView<BF16>;
    static constexpr int N = View::N;
    cg::cluster_group cluster;
    View view;
    int size, part, tid, lane, warp;
    int c0, c1, blocks, per;              // this CTA's chunks, blocks of a chunk, chunks of every CTA
    double c, c16;                        // log2(e) / temperature, 16 times that
    const double *table;                  // 2^(j / 16)
    float m;
    double unit;                          // 2^s
    u64 *list, *bins, *chunk_mass;        // (bins: the work space)
    float *chunk_max, *lane_max;          // per chunk; per chunk and lane
    unsigned *mask_words;                 // of the blocks under way
    Word *word;                           // two, in turn
    u64 *scratch;                         // kWarps + 4
    u64 *oob;                             // checking build: bounds record
    int phase;
    u64 before, mine;                     // mass of the lower parts, of this one (after a mass pass)

    __device__ __forceinline__ void barrier()
    {
        if (size > 1)
            cluster.sync();
        else
            __syncthreads();
    }
    // The end of a row that the first CTA finishes alone: it stays until nobody reads its memory any more.
    // (The others' has been read: there is a barrier behind the last exchange.)
    __device__ __forceinline__ void leave()
    {
        __syncthreads();
        if (size > 1) {
            asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
            if (part == 0)
                asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        }
    }
    // Every CTA's word, one per lane; thread 0's `w` is this CTA's.
    __device__ __forceinline__ Word exchange(const Word &w)
    {
        Word *slot = word + phase;
        phase ^= 1;
        if (tid == 0)
            *slot = w;
        barrier();
        Word r = {0.0, 0, -CUDART_INF_F, -1};
        if (lane < size)
            r = *cluster.map_shared_rank(slot, lane);
        return r;
    }
    template <class T> __device__ __forceinline__ T block_sum(T v)
    {
        v = warp_sum(v);
        T *s = reinterpret_cast<T *>(scratch);
        __syncthreads();
        if (lane == 0)
            s[warp] = v;
        __syncthreads();
        T r = s[0];
#pragma unroll
        for (int i = 1; i < kWarps; ++i)
            r += s[i];
        return r;
    }
    __device__ __forceinline__ double power(double d) const { return exp2_64(d, c16, table); }
    __device__ __forceinline__ u64 weight(float x) const
    {
        const double w = x == m ? 1.0 : power((double)x - (double)m);
        return (u64)__double2ll_rn(w * unit);
    }
    // Below which size of x the float x - reach may stand for a logit whose weight is 2^-1000, as an argument of
    // exp2_factors: its rounding, half a unit in the last place of x and reach together, is 2^-24 (10^5 + 1) < 0.6 % of
    // reach, so that the exponent stays above -1007 (10^6, with 6 %, would leave what a double's exponent holds); and
    // x - reach is finite.
    static __device__ __forceinline__ float clamp_limit(float reach) { return reach < 1e37f ? fminf(reach * 1e5f, 1e38f) : 0.f; }
    // Each warp copies its blocks into a ring of its own, STAGES ahead of the one in use; a lane reads back what
    // it copied, but for the words of the mask.  Blocks at the row's ends are read when they are used.
    static constexpr int kStage = kU * 32 * 16, kMaskWords = 32 * kU * N / 32 + 1;
    __device__ __forceinline__ bool whole(int first) const
    {
        return view.token(first) >= 0 && view.token(first) + 32 * kU * N <= view.V;
    }
    __device__ __forceinline__ void fetch(int first, char *stage, unsigned *words) const
    {
        if (whole(first)) {
            const char *from = view.row - view.head * View::ESZ + ((long long)first + lane) * 16;
            const unsigned to = (unsigned)__cvta_generic_to_shared(stage + lane * 16);
#pragma unroll
            for (int u = 0; u < kU; ++u)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + u * 512), "l"(from + u * 512) : "memory");
            if (view.mrow) {
                const int w0 = view.token(first) >> 5, last = (view.V - 1) >> 5;
                const unsigned to_w = (unsigned)__cvta_generic_to_shared(words);
                if (lane < kMaskWords && w0 + lane <= last)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to_w + lane * 4), "l"(view.mrow + w0 + lane) : "memory");
                if (kMaskWords > 32 && view.head != 0 && lane == 0 && w0 + 32 <= last)      // (bf16: the 33rd word)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to_w + 128), "l"(view.mrow + w0 + 32) : "memory");
            }
        }
    }
    __device__ __forceinline__ void take(int first, const char *stage, const unsigned *words, uint4 (&raw)[kU]) const
    {
        if (whole(first)) {
            const uint4 *from = reinterpret_cast<const uint4 *>(stage) + lane;
#pragma unroll
            for (int u = 0; u < kU; ++u)
                raw[u] = from[u * 32];
            if (view.mrow && view.head == 0) {
                const unsigned *w = words + (lane * N >> 5);
#pragma unroll
                for (int u = 0; u < kU; ++u)
                    raw[u] = View::mask(raw[u], w[u * N] >> (lane * N & 31));
            } else if (view.mrow) {
                const int at = (view.token(first) & 31) + lane * N;
                const unsigned *w = words + (at >> 5);
#pragma unroll
                for (int u = 0; u < kU; ++u)
                    raw[u] = View::mask(raw[u], __funnelshift_r(w[u * N], w[u * N + 1], at & 31));
            }
        } else {
#pragma unroll
            for (int u = 0; u < kU; ++u)
                raw[u] = view.masked(first + u * 32 + lane);
        }
    }
    // use(raw, first vector) for every block of this warp's chunks, close(chunk) behind each chunk.  `ring`: STAGES
    // blocks for each warp; whoever used that memory before has passed a barrier.
    template <int STAGES, class U, class C> __device__ __forceinline__ void stream(void *ring, U use, C close)
    {
        char *stage = reinterpret_cast<char *>(ring) + warp * STAGES * kStage;
        unsigned *words = mask_words + warp * 2 * (kMaskWords + 3);
        int ch = c0 + warp, i = 0;                       // the block to use: the i-th of chunk ch
        int ch2 = ch, i2 = 0;                            // the block to fetch
        auto next = [&](int s) {
            if (ch2 < c1)
                fetch((ch2 * blocks + i2) * 32 * kU, stage + s * kStage, words + s * (kMaskWords + 3));
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (++i2 == blocks) {
                i2 = 0;
                ch2 += kWarps;
            }
        };
#pragma unroll
        for (int s = 0; s < STAGES; ++s)
            next(s);
#pragma unroll 1
        for (int s = 0; ch < c1; s = STAGES == 2 ? s ^ 1 : 0) {
            const int first = (ch * blocks + i) * 32 * kU;
            uint4 raw[kU];
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            __syncwarp();
            take(first, stage + s * kStage, words + s * (kMaskWords + 3), raw);
            __syncwarp();
            next(s);
            use(raw, first);
            if (++i == blocks) {
                close(ch);
                i = 0;
                ch += kWarps;
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
    }
    // f(raw vector, token of its first logit) for every vector of this CTA's chunks, close(chunk) behind each chunk.
    // One vector's code, run kU times: a pass that a row takes once costs what its code takes to come.
    template <class F, class C> __device__ __forceinline__ void each_vector(void *ring, F f, C close)
    {
        stream<1>(ring, [&](uint4 (&raw)[kU], int first) {
#pragma unroll 1
            for (int u = 0; u < kU; ++u) {
                f(raw[0], view.token(first + u * 32 + lane));
#pragma unroll
                for (int i = 1; i < kU; ++i)
                    raw[i - 1] = raw[i];
            }
        }, close);
    }
    // f(logit, token) for every allowed logit above -infinity
    template <class F, class C> __device__ __forceinline__ void each(void *ring, F f, C close)
    {
        each_vector(ring, [&](const uint4 &raw, int tok) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = View::plain(raw, e);
                if (x > -CUDART_INF_F)                   // (and no NaN)
                    f(x, tok + e);
            }
        }, close);
    }
    // Maximum of every lane's logits in a chunk, maximum of the chunk and its sum of 2^(c (x - maximum)) as the
    // bits of a double: taken in 32 bits, or in 64.
    enum { kMaximum, kSum32, kSum64 };
    template <int WHAT> __device__ __forceinline__ void first_pass()
    {
        const float c32 = (float)c, reach = (float)(1000.0 / c), limit = clamp_limit(reach);
        const double k16 = c16;
        float top = -CUDART_INF_F;
        float2 s32 = {0.f, 0.f};
        double s64 = 0.0;
        auto use = [&](uint4 (&raw)[kU], int) {
            float t = -CUDART_INF_F;
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int e = 0; e < N; e += 2)
                    t = max3(t, View::plain(raw[u], e), View::plain(raw[u], e + 1));
            if (WHAT == kMaximum)
                top = fmaxf(top, t);
            if (WHAT == kSum32) {
                if (t > top) {
                    const float f = exp2_fast((top - t) * c32);
                    s32.x *= f;
                    s32.y *= f;
                    top = t;
                }
                const float ref = top == -CUDART_INF_F ? 0.f : top;
#pragma unroll
                for (int u = 0; u < kU; ++u)
#pragma unroll
                    for (int e = 0; e < N; e += 2)
                        add_exponentials(s32, View::plain(raw[u], e), View::plain(raw[u], e + 1), ref, c32);
            }
            if (WHAT == kSum64) {
                if (t > top) {
                    s64 *= top == -CUDART_INF_F ? 0.0 : power((double)top - (double)t);
                    top = t;
                }
                // logits far below (and NaN) add 2^-1000 or so - where floats are fine enough to say that
                const float least = top - reach;
                if (!(fabsf(top) < limit)) {
                    for (int u = 0; u < kU * N && top > -CUDART_INF_F; ++u) {
                        const float x = View::value(raw[u / N], u % N);
                        s64 += x == top ? 1.0 : power((double)x - (double)top);
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < kU; ++u)
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const double2 f = exp2_factors((double)fmaxf(View::plain(raw[u], e), least) - (double)top, k16, table);
                            s64 = fma(f.x, f.y, s64);
                        }
                }
            }
        };
        auto close = [&](int ch) {
            lane_max[(ch - c0) * 32 + lane] = top;
            const float most = warp_max(top);
            double sum = 0.0;
            if (WHAT == kSum32) {
                float s = (s32.x + s32.y) * exp2_fast(top == most ? 0.f : (top - most) * c32);
#pragma unroll
                for (int off = 16; off > 0; off >>= 1)
                    s += __shfl_xor_sync(kFull, s, off);
                sum = s;
            }
            if (WHAT == kSum64 && top > -CUDART_INF_F)
                sum = s64 * power((double)top - (double)most);
            const bool again = most == CUDART_INF_F || __any_sync(kFull, sum != sum);
            if (again) {
                // NaN adds nothing, infinite logits share the sum
                sum = 0.0;
                for (int v = ch * blocks * kU * 32 + lane; v < (ch + 1) * blocks * kU * 32; v += 32) {
                    const uint4 raw = view.masked(v);
                    for (int e = 0; e < N; ++e) {
                        const float x = View::value(raw, e);
                        sum += x == most ? 1.0 : x == -CUDART_INF_F ? 0.0 : power((double)x - (double)most);
                    }
                }
            }
            if (WHAT == kSum64 || again)
                sum = warp_sum(sum);
            if (lane == 0) {
                chunk_max[ch - c0] = most;
                chunk_mass[ch - c0] = (u64)__double_as_longlong(sum);
            }
            top = -CUDART_INF_F;
            s32 = {0.f, 0.f};
            s64 = 0.0;
        };
        stream<2>(list, use, close);
    }
    // This CTA's and the row's sums of the chunks' masses; returns the row's.
    __device__ __forceinline__ u64 share_masses()
    {
        u64 s = 0;
        for (int i = tid; i < c1 - c0; i += kThreads)
            s += chunk_mass[i];
        mine = block_sum(s);
        const Word r = exchange({0.0, mine, 0.f, 0});
        before = warp_sum(lane < part ? r.mass : 0);
        return warp_sum(lane < size ? r.mass : 0);
    }
    // Sums of f(logit, token) by chunk; returns the row's.
    template <class F> __device__ __forceinline__ u64 mass_pass(F f)
    {
        u64 s = 0;
        each(list, [&](float x, int tok) { s += f(x, tok); }, [&](int ch) {
            s = warp_sum(s);
            if (lane == 0)
                chunk_mass[ch - c0] = s;
            s = 0;
        });
        return share_masses();
    }
    // After a mass pass over f: the first token by id whose running sum exceeds t, in warp 0 of the CTA
    // that holds it, -1 everywhere else.
    template <class F> __device__ __forceinline__ int find(F f, u64 t)
    {
        if (warp != 0 || t < before || t >= before + mine)
            return -1;
        u64 base = before;
        int ch = c0;
        for (;; ch += 32) {                              // (ends: the sum of all chunks exceeds t)
            const u64 w = ch + lane < c1 ? chunk_mass[ch - c0 + lane] : 0;
            const u64 upto = base + inclusive_scan(w, lane);
            const unsigned over = __ballot_sync(kFull, upto > t);
            if (over) {
                const int l = __ffs((int)over) - 1;
                base = __shfl_sync(kFull, upto - w, l);
                ch += l;
                break;
            }
            base = __shfl_sync(kFull, upto, 31);
            if (ch + 32 >= c1)
                break;
        }
        int last = -1, first = kNone;                    // last token with any weight, first with the largest logit
        float top = -CUDART_INF_F;
        for (int v = ch * blocks * kU * 32 + lane; v < (ch + 1) * blocks * kU * 32; v += 32) {
            const uint4 raw = view.masked(v);
            u64 s = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = View::value(raw, e);
                const u64 w = x > -CUDART_INF_F ? f(x, view.token(v) + e) : 0;
                s += w;
                last = w ? view.token(v) + e : last;
                if (x > top) {
                    top = x;
                    first = view.token(v) + e;
                }
            }
            const u64 upto = base + inclusive_scan(s, lane);
            const unsigned over = __ballot_sync(kFull, upto > t);
            if (over) {
                const int l = __ffs((int)over) - 1;
                u64 at = upto - s;
                int tok = -1;
                for (int e = 0; e < N; ++e) {
                    const float x = View::value(raw, e);
                    at += x > -CUDART_INF_F ? f(x, view.token(v) + e) : 0;
                    if (tok < 0 && at > t)
                        tok = view.token(v) + e;
                }
                return __shfl_sync(kFull, tok, l);
            }
            base = __shfl_sync(kFull, upto, 31);
        }
        // The chunk's mass and its tokens' differ by rounding where the former is a sum of unrounded weights: the last
        // token, or where all weights round to nothing the chunk's first in the row's order, which is kept if any is.
        last = __reduce_max_sync(kFull, last);
        const float most = warp_max(top);
        first = __reduce_min_sync(kFull, top == most ? first : kNone);
        return last >= 0 ? last : first;
    }
    // Distance from the maximum as one of kBins numbers, ascending: 32 to an octave from 2^-6 on.
    static constexpr int kFirstBin = ((127 - 6) << 5) - 1;
    __device__ __forceinline__ int bin_of(float x) const
    {
        if (x == m)
            return 0;
        const int b = (int)(__float_as_uint(m - x) >> 18) - kFirstBin;
        return min(max(b, 1), kBins - 1);
    }
    // Of two bins a thread: the first at which their running sum reaches target, what lies before it and its own
    // go to scratch[kWarps ..] (all ones: none does).
    __device__ __forceinline__ void cross(const u64 (&w)[2], u64 target)
    {
        const u64 s = w[0] + w[1], upto = inclusive_scan(s, lane);
        if (lane == 31)
            scratch[warp] = upto;
        if (tid == 0)
            scratch[kWarps] = ~0ull;
        __syncthreads();
        u64 base = upto - s;
#pragma unroll
        for (int i = 0; i < kWarps - 1; ++i)
            base += i < warp ? scratch[i] : 0;
        if (base < target && base + s >= target) {
            const int second = base + w[0] < target;
            scratch[kWarps] = tid * 2 + second;
            scratch[kWarps + 1] = base + (second ? w[0] : 0);
            scratch[kWarps + 2] = second ? w[1] : w[0];
        }
        __syncthreads();
    }
    // The cluster's sums of two bins a thread (counted in T), after a barrier; the bins may be changed behind another.
    template <class T> __device__ __forceinline__ void merge_bins(u64 (&w)[2], int set = 0)
    {
        barrier();
        w[0] = w[1] = 0;
        for (int r = 0; r < size; ++r) {
            const T *o = cluster.map_shared_rank(reinterpret_cast<T *>(bins), r) + set * kBins + tid * 2;
            w[0] += o[0];
            w[1] += o[1];
        }
    }
    template <class T, class F> __device__ __forceinline__ void fill_bins(F f, int set = 0)     // f(logit, token, bin): weight, 0: none
    {
        T *to = reinterpret_cast<T *>(bins) + set * kBins;
        to[tid * 2] = to[tid * 2 + 1] = 0;
        __syncthreads();
        each(list, [&](float x, int tok) {
            int bin;
            const T w = f(x, tok, bin);
            if (w)
                atomicAdd(to + bin, w);
        }, [](int) {});
    }
    // The ordered bits that the logits of bins b1 .. b2 can have: lo + [0, 2^bits).  They lie within m - [d0, d1],
    // widened by the difference's rounding.
    __device__ __forceinline__ void range_of(int b1, int b2, unsigned &lo, int &bits) const
    {
        const float d0 = b1 <= 1 ? 0.f : __uint_as_float((unsigned)(b1 + kFirstBin) << 18) * (1.f - 0x1p-22f);
        const float d1 = b2 == kBins - 1 ? CUDART_INF_F : __uint_as_float((unsigned)(b2 + 1 + kFirstBin) << 18) * (1.f + 0x1p-22f);
        const unsigned least = order_of(-CUDART_INF_F);
        lo = b1 == 0 ? order_of(m) : max(order_of(m), order_of(m - d0) - 2);
        const unsigned hi = b2 == 0 ? lo : m == CUDART_INF_F ? least : min(order_of(m - d1) + 2, least);
        bits = hi > lo ? 32 - __clz((int)(hi - lo)) : 0;
    }
    // The least finite logit with ordered bits lo + [0, 2^bits)
    static __device__ __forceinline__ float lowest(unsigned lo, int bits)
    {
        return logit_of((unsigned)min((u64)lo + ((u64)1 << bits) - 1, (u64)order_of(-FLT_MAX)));
    }
    // The shortest prefix of the row's order whose sum of f, together with `sum` for the logits before them,
    // reaches target, among the logits `in` with ordered bits lo + [0, 2^bits): by kDigit digits at a time.
    // false: they do not.  Equal logits have equal f.
    template <class T, class F, class P>
    __device__ __forceinline__ bool digits(F f, P in, u64 target, u64 sum, unsigned lo, int bits, Cut &cut)
    {
        u64 at = 0;
        do {
            const int shift = max(bits - kDigit, 0);
            const float high = logit_of(lo), low = lowest(lo, bits);
            fill_bins<T>([&](float x, int tok, int &bin) {
                if (x > high || x < low || !in(x))
                    return (T)0;
                bin = (int)((order_of(x) - lo) >> shift);
                return f(x, tok);
            });
            u64 w[2];
            merge_bins<T>(w);
            cross(w, target - sum);
            const u64 digit = scratch[kWarps];
            sum += digit == ~0ull ? 0 : scratch[kWarps + 1];
            at = scratch[kWarps + 2];
            barrier();
            if (digit == ~0ull)
                return false;
            lo += (unsigned)digit << shift;
            bits = shift;
        } while (bits > 0);
        cut.x = logit_of(lo);
        cut.last = kNone;
        const u64 one = f(cut.x, 0), r = (target - sum + one - 1) / one;      // equal logits that are kept
        if (r * one < at) {
            const float x = cut.x;
            auto tie = [x](float v, int) { return (u64)(v == x); };
            mass_pass(tie);
            cut.last = everybody(find(tie, r - 1));
        }
        return true;
    }
    // ... of the whole row: first by distance from the maximum, which spreads the logits over the bins.
    template <class T, class F> __device__ __forceinline__ bool select(F f, u64 target, Cut &cut)
    {
        fill_bins<T>([&](float x, int tok, int &bin) {
            bin = bin_of(x);
            return f(x, tok);
        });
        u64 w[2];
        merge_bins<T>(w);
        cross(w, target);
        const u64 b = scratch[kWarps], sum = scratch[kWarps + 1];
        barrier();
        if (b == ~0ull)
            return false;
        unsigned lo;
        int bits;
        range_of((int)b, (int)b, lo, bits);
        return digits<T>(f, [&](float x) { return bin_of(x) == (int)b; }, target, sum, lo, bits, cut);
    }
    // Ordered bits [o1, o2] within which the sum of the weights reaches target, by weights in 32 bits as whole
    // numbers of 2^-31 of their sum `total` (two sets of bins, to be changed behind a barrier).  These are off by half a number each and by 2^-18 of all (arguments of
    // exponentials): what is that near to the target is within.  Nothing relies on it.
    __device__ __forceinline__ void narrow(double total, u64 target, unsigned &o1, unsigned &o2)
    {
        const float c32 = (float)c, k = (float)(0x1p+31 / total);
        const u64 want = (u64)((double)target / unit / total * 0x1p+31), slack = 65536 + view.V / 2;
        const u64 from = want > slack ? want - slack : 1, to = want + slack;
        auto about = [&](float x) { return __float2uint_rn((x == m ? 1.f : exp2_fast((x - m) * c32)) * k); };
        o1 = 1;
        o2 = 0;
        u64 w[2];
        fill_bins<unsigned>([&](float x, int, int &bin) {
            bin = bin_of(x);
            return about(x);
        });
        merge_bins<unsigned>(w);
        cross(w, from);
        const u64 b1 = scratch[kWarps], sum = scratch[kWarps + 1];
        __syncthreads();
        cross(w, to);
        const int b2 = (int)min(scratch[kWarps], (u64)kBins - 1);
        if (b1 == ~0ull)
            return;
        unsigned lo;
        int bits;
        range_of((int)b1, b2, lo, bits);
        const int shift = max(bits - kDigit, 0);
        const float high = logit_of(lo), low = lowest(lo, bits);
        fill_bins<unsigned>([&](float x, int, int &bin) {
            if (x > high || x < low)
                return 0u;
            const int b = bin_of(x);
            bin = (int)((order_of(x) - lo) >> shift);
            return b >= (int)b1 && b <= b2 ? about(x) : 0u;
        }, 1);
        merge_bins<unsigned>(w, 1);
        cross(w, from - sum);
        const u64 d1 = scratch[kWarps];
        __syncthreads();
        cross(w, to - sum);
        const u64 d2 = min(scratch[kWarps], (u64)kBins - 1);
        if (d1 == ~0ull)
            return;
        o1 = lo + (unsigned)(d1 << shift);
        o2 = (unsigned)min((u64)lo + ((d2 + 1) << shift) - 1, (u64)0xffffffffu);
    }
    // The chunks' masses of the logits above ordered bits o1 - their sum is returned -, those within [o1, o2] into
    // the list of the cluster's first CTA, `found` of them.  (count is 0, and the barrier behind that has been passed.)
    __device__ __forceinline__ u64 split(unsigned o1, unsigned o2, int *count, int &found)
    {
        bool full = false;
        const float high = logit_of(o1), low = logit_of(min(o2, order_of(-FLT_MAX)));
        // (what is not above adds 2^-1000 or so, where floats are fine enough to say that)
        const float reach = (float)(1000.0 / c), least = m - reach;
        const bool fine = fabsf(m) < clamp_limit(reach);
        double s = 0.0;
        each_vector(bins, [&](const uint4 &raw, int tok) {
            unsigned near = 0;                           // logits around the border
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = View::plain(raw, e);
                const double d = (double)(x > high ? x : least) - (double)m;
                if (fine) {
                    const double2 f = exp2_factors(d, c16, table);
                    s = fma(f.x, f.y, s);
                } else if (x > high)
                    s += x == m ? 1.0 : power(d);
                near |= x <= high && x >= low ? 1u << e : 0u;
            }
            for (; near; near &= near - 1) {
                const int e = __ffs((int)near) - 1;
                collect(View::at(raw, e), tok + e, count, full);
            }
        }, [&](int ch) {
            s = warp_sum(s);
            if (lane == 0)
                chunk_mass[ch - c0] = (u64)__double2ll_rn(s * unit);
            s = 0.0;
        });
        found = collected(count);
        return share_masses();
    }
    // Running sums of the weights of the list's first n entries, kThreads of them at a time, into the work space.
    __device__ __forceinline__ void running_sums(int n)
    {
        u64 base = 0;
        for (int i0 = 0; i0 < n; i0 += kThreads) {
            const int i = i0 + tid;
            const u64 w = i < n ? weight(logit_of((unsigned)(list[i] >> 32))) : 0;
            const u64 upto = inclusive_scan(w, lane);
            __syncthreads();
            if (lane == 31)
                scratch[warp] = upto;
            __syncthreads();
            u64 below = base;
#pragma unroll
            for (int j = 0; j < kWarps; ++j) {
                below += j < warp ? scratch[j] : 0;
                base += scratch[j];
            }
            if (i < n)
                bins[i] = below + upto;
        }
        __syncthreads();
    }
    // Entries up to the first whose running sum reaches target (all n where none does).
    __device__ __forceinline__ int reached_by(u64 target, int n) const
    {
        int lo = 0, hi = n - 1;                          // (every thread looks for itself)
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (bins[mid] >= target)
                hi = mid;
            else
                lo = mid + 1;
        }
        return lo + 1;
    }
    // The cut at which the row's mass reaches target, and what it keeps; afterwards the chunks' masses are those of
    // the kept tokens.  Most of the row is counted as a whole, the logits around the border one by one.
    __device__ __forceinline__ u64 cut_mass(double total, u64 target, int *count, Cut &cut)
    {
        unsigned o1, o2;
        narrow(total, target, o1, o2);
        if (tid == 0)
            *count = 0;
        barrier();
        int found;
        const u64 above = split(o1, o2, count, found);
        Word w = {0.0, 0, 0.f, 0};
        if (found <= kList && part == 0 && found > 0 && above < target) {
            sort_list(list, found);
            running_sums(found);
            if (above + bins[found - 1] >= target) {
                const int n = reached_by(target - above, found);
                w = {0.0, above + bins[n - 1], logit_of((unsigned)(list[n - 1] >> 32)), (int)(unsigned)list[n - 1]};
                for (int i = tid; i < n; i += kThreads) {
                    const int ch = ((int)(unsigned)list[i] + view.head) / N / (32 * kU) / blocks, owner = ch / per;
                    if (CSTR_INB(oob, owner, size, CSTR_SITE_SAMPLE))
                        atomicAdd(cluster.map_shared_rank(chunk_mass + ch - owner * per, owner), bins[i] - (i ? bins[i - 1] : 0));
                }
            }
        }
        w = exchange(w);                                 // (the first CTA's)
        const u64 kept = __shfl_sync(kFull, w.mass, 0);
        cut.x = __shfl_sync(kFull, w.m, 0);
        cut.last = __shfl_sync(kFull, w.token, 0);
        if (kept) {
            share_masses();
            return kept;
        }
        // many equal logits at the border (or, never seen, a border outside)
        auto f = [&](float x, int) { return weight(x); };
        const int bits = o2 > o1 ? 32 - __clz((int)(o2 - o1)) : 0;
        const float low = logit_of(min(o2, order_of(-FLT_MAX)));
        if (!(found > kList && above < target && digits<u64>(f, [&](float x) { return x >= low; }, target, above, o1, bits, cut)) &&
            !select<u64>(f, target, cut))
            cut = {-CUDART_INF_F, kNone};
        return mass_pass([&](float x, int tok) { return cut.keeps(x, tok) ? weight(x) : (u64)0; });
    }
    // The lowest bin up to which f, summed over the lanes' maxima of the whole row, reaches `target`; the
    // last bin where the row does not.  Every lane's maximum is a logit of its own, so that so much lies
    // in the bins up to that one at least.
    template <class F> __device__ __forceinline__ int reach(F f, u64 target, bool &reached)
    {
        unsigned *hist = reinterpret_cast<unsigned *>(bins);     // zero since the kernel began
        for (int i = tid; i < (c1 - c0) * 32; i += kThreads) {
            const float x = lane_max[i];
            const unsigned w = x > -CUDART_INF_F ? f(x) : 0u;
            if (w)
                atomicAdd(hist + bin_of(x), w);
        }
        barrier();
        u64 w[2] = {0, 0};
        for (int r = 0; r < size; ++r) {
            const uint2 o = reinterpret_cast<const uint2 *>(cluster.map_shared_rank(hist, r))[tid];
            w[0] += o.x;
            w[1] += o.y;
        }
        cross(w, target);
        const u64 b = scratch[kWarps];
        reached = b != ~0ull;
        return reached ? (int)b : kBins - 1;
    }
    // Entries of the row's list, the first CTA's: each CTA collects its own, whose number is in count[0], and the
    // others' go there in one piece.  (A remote counter answers in a microsecond.)
    __device__ __forceinline__ void collect(float x, int tok, int *count, bool &full)
    {
        const int at = full ? kList : atomicAdd(count, 1);
        full = at >= kList;
        if (!full)
            list[at] = ((u64)order_of(x) << 32) | (unsigned)tok;
    }
    // Returns how many there are (more than kList: the list is not whole); the counters are behind a barrier.
    __device__ __forceinline__ int collected(int *count)
    {
        __syncthreads();
        int *all = cluster.map_shared_rank(count, 0);
        if (part != 0 && *count > 0) {
            const int n = min(*count, kList);
            if (tid == 0)
                scratch[0] = (u64)atomicAdd(all, *count);
            __syncthreads();
            const long long at = (long long)scratch[0];
            u64 *to = cluster.map_shared_rank(list, 0);
            for (int i = tid; i < n; i += kThreads)
                if (at + i < kList)
                    to[at + i] = list[i];
        }
        barrier();
        return *all;
    }
    // Logits of the row in bins up to `last`, as (order, token), into the list; returns how many there are.
    __device__ __forceinline__ int gather(int last, int *count, int *hits)
    {
        // the lanes to look at, then all threads share their vectors
        unsigned short *lanes = reinterpret_cast<unsigned short *>(bins + kList / 2);
        for (int i = tid; i < (c1 - c0) * 32; i += kThreads)
            if (lane_max[i] > -CUDART_INF_F && bin_of(lane_max[i]) <= last)
                lanes[atomicAdd(hits, 1)] = (unsigned short)i;
        __syncthreads();
        bool full = false;
        const int each = blocks * kU, units = *hits * each;
#pragma unroll 2
        for (int q = tid; q < units; q += kThreads) {
            const int h = q / each, i = lanes[h];
            const int v = ((c0 + (i >> 5)) * each + (q - h * each)) * 32 + (i & 31);
            const uint4 raw = view.masked(v);
            unsigned near = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = View::value(raw, e);
                near |= x > -CUDART_INF_F && bin_of(x) <= last ? 1u << e : 0u;
            }
            for (; near; near &= near - 1) {
                const int e = __ffs((int)near) - 1;
                collect(View::at(raw, e), view.token(v) + e, count, full);
            }
        }
        return collected(count);
    }
    // The largest of the CTAs' (warp 0's) tokens, for all
    __device__ __forceinline__ int everybody(int tok)
    {
        const Word r = exchange({0.0, 0, 0.f, tok});
        return __reduce_max_sync(kFull, r.token);
    }
};

// The token of a row whose `found` candidates are in the list of this CTA: the tokens below `low` and
// beyond top_k leave, then top_p of `whole` (0: of what is left) is kept.  done(token, logit, kept mass) by one thread.
template <bool BF16, class F>
__device__ __forceinline__ void from_list(Row<BF16> &r, int found, int top_k, float low, float top_p, u64 whole, float u, int *count,
                                          F done)
{
    const int tid = r.tid, lane = r.lane, warp = r.warp;
    if (found <= kThreads) {
        // Each entry is compared with all others by as many threads as there are for it: its rank, what lies
        // before it, then - of those that are kept - what its id and lower ones hold.
        int share = 1;
        while (share < 8 && found * share * 2 <= kThreads)
            share *= 2;
        const int at = tid / share, sub = tid & (share - 1);
        const bool in = at < found;
        const u64 key = in ? r.list[at] : ~0ull;
        const float x = logit_of((unsigned)(key >> 32));
        u64 w = in ? r.weight(x) : 0;
        if (in && sub == 0)
            r.bins[at] = w;
        __syncthreads();
        int rank = 0;
        u64 before = 0;
        if (warp * 32 < found * share) {
            for (int j = sub; j < found; j += share) {
                const bool first = r.list[j] < key;
                rank += first;
                before += first ? r.bins[j] : 0;
            }
            for (int off = 1; off < share; off *= 2) {
                rank += __shfl_xor_sync(kFull, rank, off);
                before += __shfl_xor_sync(kFull, before, off);
            }
        }
        // (the first token is kept in any case: min_p is at most 1, top_k at least 2, the target above 0)
        bool keep = in && x >= low && (top_k <= 0 || rank < top_k);
        if (top_p < 1.f) {
            const u64 target = part_of(whole ? whole : r.block_sum(keep && sub == 0 ? w : 0), top_p, true);
            keep = keep && before < target;
        }
        w = keep ? w : 0;
        const u64 kept = r.block_sum(sub == 0 ? w : 0), t = part_of(kept, u, false);
        __syncthreads();
        if (in && sub == 0)
            r.bins[at] = w;
        __syncthreads();
        const unsigned id = (unsigned)key;
        u64 upto = 0;
        if (warp * 32 < found * share) {
            for (int j = sub; j < found; j += share)
                upto += (unsigned)r.list[j] <= id ? r.bins[j] : 0;
            for (int off = 1; off < share; off *= 2)
                upto += __shfl_xor_sync(kFull, upto, off);
        }
        if (keep && sub == 0 && upto > t && upto - w <= t)
            done((int)id, x, kept);
        return;
    }
    sort_list(r.list, found);
    if (tid == 0)
        *count = 0;
    __syncthreads();
    // the cuts by rank and by logit keep a prefix
    int n = 0;
    for (int i = tid; i < found; i += kThreads)
        n += logit_of((unsigned)(r.list[i] >> 32)) >= low;
    n = __reduce_add_sync(kFull, n);
    if (lane == 0 && n)
        atomicAdd(count, n);
    __syncthreads();
    n = min(*count, top_k > 0 ? min(top_k, found) : found);
    r.running_sums(n);
    if (top_p < 1.f)                                     // the first whose running sum reaches the target ends the prefix
        n = r.reached_by(part_of(whole ? whole : r.bins[n - 1], top_p, true), n);
    const u64 kept = r.bins[n - 1], t = part_of(kept, u, false);
    // by id: bit by bit, is the sum over the ids below the next half above t?
    auto weight_at = [&](int i) { return r.bins[i] - (i ? r.bins[i - 1] : 0); };
    unsigned id = 0;
    u64 below = 0;
    for (int bit = 22; bit >= 0; --bit) {
        u64 s = 0;
        for (int i = tid; i < n; i += kThreads)
            s += ((unsigned)r.list[i] >> bit) == id << 1 ? weight_at(i) : 0;
        s = r.block_sum(s);
        const bool upper = below + s <= t;
        below += upper ? s : 0;
        id = id << 1 | (upper ? 1u : 0u);
    }
    for (int i = tid; i < n; i += kThreads)
        if ((unsigned)r.list[i] == id)
            done((int)id, logit_of((unsigned)(r.list[i] >> 32)), kept);
}

template <bool BF16, bool TOP>
__global__ void __launch_bounds__(kThreads, 4)
sample_kernel(const __grid_constant__ SampleParams p)
{
    using View = RowView<BF16>;
    constexpr int N = View::N;
    extern __shared__ __align__(16) u64 s_dynamic[];      // list, bins, then masses and maxima of the chunks
    __shared__ Word s_word[2];
    __shared__ u64 s_scratch[kWarps + 4];
    __shared__ float s_max[kWarps];
    __shared__ double s_table[16];
    __shared__ unsigned s_mask[kWarps * 2 * (Row<BF16>::kMaskWords + 3)];
    __shared__ int s_count, s_left, s_hits;
    static_assert(kBins == 2 * kThreads && kBins * 8 <= kList * 4 && kMaxChunks * 32 * 2 <= kList * 4, "bins and lanes share the work space");
    static_assert(kWarps * 2 * Row<BF16>::kStage <= 2 * kList * 8, "the ring lies in list and work space");
    cstr_wait_for_earlier_kernels();
    cstr_let_next_kernel_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int size = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / size;
    int table, state;
    const uint32_t *mrow;
    bool active = row_state(p.t, row, table, state, mrow);

    // the row's settings
    float u = 0.f, top_p = 1.f, min_p = 0.f;
    int top_k = 0;
    double c = p.c;
    bool cold = false;                                   // temperature 0
    if (!TOP) {
        const float temperature = p.temperature ? p.temperature[row] : 1.f;
        u = p.uniform[row];
        top_p = p.top_p ? p.top_p[row] : 1.f;
        min_p = p.min_p ? p.min_p[row] : 0.f;
        top_k = p.top_k ? p.top_k[row] : 0;
        cold = temperature == 0.f;
        c = cold ? 1.0 : 1.4426950408889634 / (double)temperature;
        if (!(temperature >= 0.f) || temperature == CUDART_INF_F || !((float)c < CUDART_INF_F) || u != u ||
            top_p != top_p || min_p != min_p)
            active = false;
        u = fminf(fmaxf(u, 0.f), 0x1.fffffep-1f);
    }
    // (the state's number in the table, before it is needed)
    const int inner = !TOP && p.t.n > 0 && active && p.t.tab[table].rank ? p.t.tab[table].rank[state] : state;
    // token and state of a row, by one thread
    auto finish = [&](int token, float logp, float kept) {
        int next = CSTR_DEAD;
        if (token >= 0 && p.t.n > 0 && CSTR_INB(p.oob, token, p.V, CSTR_SITE_SAMPLE))
            next = next_state(p.t.tab[table], inner, token);
        p.tokens[row] = token;
        if (p.states_out)
            p.states_out[row] = next;
        if (p.logp)
            p.logp[row] = logp;
        if (p.kept)
            p.kept[row] = kept;
        if (p.accept_out)
            p.accept_out[row] = next >= 0 ? (uint8_t)(p.t.tab[table].accept[next] != 0) : (uint8_t)0;
    };
    if (!active) {
        if (part == 0) {
            if (TOP) {
                for (int i = tid; i < p.n; i += kThreads) {
                    p.ids[(long long)row * p.n + i] = -1;
                    p.logp[(long long)row * p.n + i] = -CUDART_INF_F;
                }
                if (tid == 0 && p.lse)
                    p.lse[row] = -CUDART_INF_F;
            } else if (tid == 0)
                finish(-1, -CUDART_INF_F, 0.f);
        }
        return;
    }

    Row<BF16> r = {cluster, View(p.logits, (long long)row * p.ld, p.V, mrow), size, part, tid, lane, warp};
    r.blocks = p.blocks;
    const int chunks = (r.view.vectors() + 32 * kU * p.blocks - 1) / (32 * kU * p.blocks), per = (chunks + size - 1) / size;
    r.per = per;
    r.c0 = min(part * per, chunks);
    r.c1 = min(r.c0 + per, chunks);
    r.c = c;
    r.c16 = 16.0 * c;
    r.table = s_table;
    r.unit = __hiloint2double((1023 + p.scale_bits) << 20, 0);
    r.list = s_dynamic;
    r.bins = s_dynamic + kList;
    r.chunk_mass = r.bins + kList;
    r.chunk_max = reinterpret_cast<float *>(r.chunk_mass + p.per);
    r.lane_max = r.chunk_max + p.per;
    r.mask_words = s_mask;
    r.word = s_word;
    r.scratch = s_scratch;
    r.oob = p.oob;
    r.phase = 0;
    if (tid == 0)
        s_count = s_hits = 0;
    if (tid < 16)
        s_table[tid] = exp2((double)tid / 16.0);
    __syncthreads();

    // One pass over memory.  Where the whole sum decides about the token it is taken in 64 bits.
    const bool plain = !TOP && !cold && top_k <= 0 && top_p >= 1.f && min_p <= 0.f;
    const bool exact_sum = plain || (!TOP && !cold && top_k <= 0 && top_p < 1.f && min_p <= 0.f);
    const float c32 = (float)c;
    if (!TOP && cold)
        r.template first_pass<Row<BF16>::kMaximum>();
    else if (!TOP && exact_sum)
        r.template first_pass<Row<BF16>::kSum64>();
    else
        r.template first_pass<Row<BF16>::kSum32>();
    reinterpret_cast<uint2 *>(r.bins)[tid] = make_uint2(0u, 0u);        // counts of 32 bits
    auto chunk_sum = [&](int i, float ref) {              // relative to ref
        const float top = r.chunk_max[i];
        const double s = __longlong_as_double((long long)r.chunk_mass[i]);
        return top == ref ? s : s * r.power((double)top - (double)ref);
    };
    // every warp its own chunks, then all of the CTA's
    float m = -CUDART_INF_F;
    for (int i = warp + lane * kWarps; i < r.c1 - r.c0; i += 32 * kWarps)
        m = fmaxf(m, r.chunk_max[i]);
    m = warp_max(m);
    double sum = 0.0;
    if (m > -CUDART_INF_F)
        for (int i = warp + lane * kWarps; i < r.c1 - r.c0; i += 32 * kWarps)
            sum += chunk_sum(i, m);
    sum = warp_sum(sum);
    if (lane == 0) {
        s_scratch[warp] = (u64)__double_as_longlong(sum);
        s_max[warp] = m;
    }
    __syncthreads();
    m = s_max[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i)
        m = fmaxf(m, s_max[i]);
    sum = 0.0;
    if (lane < kWarps && m > -CUDART_INF_F) {
        const double s = __longlong_as_double((long long)s_scratch[lane]);
        sum = s_max[lane] == m ? s : s * r.power((double)s_max[lane] - (double)m);
    }
    sum = warp_sum(sum);
    const Word all = r.exchange({sum, 0, m, 0});
    const float own_max = m;
    m = warp_max(lane < size ? all.m : -CUDART_INF_F);
    r.m = m;
    double total = 0.0;                                   // of the row, relative to m
    if (lane < size && all.sum > 0.0)
        total = all.m == m ? all.sum : all.sum * r.power((double)all.m - (double)m);
    total = warp_sum(total);

    if (TOP) {
        if (tid == 0 && part == 0 && p.lse)
            p.lse[row] = m == -CUDART_INF_F ? m : (float)((double)m * c * 0.6931471805599453 + log(total));
        int found = 0;
        if (m == -CUDART_INF_F)
            r.barrier();                                  // (the words have been read)
        else {
            bool reached;
            found = r.gather(r.reach([](float) { return 1u; }, (u64)p.n, reached), &s_count, &s_hits);
            if (found > kList) {                          // many equal logits, or more tokens than half the lanes
                Cut cut = {-CUDART_INF_F, kNone};
                r.template select<unsigned>([](float, int) { return 1u; }, (u64)p.n, cut);
                if (tid == 0)
                    s_count = 0;
                r.barrier();
                bool full = false;
                r.each(r.bins, [&](float x, int tok) {
                    if (cut.keeps(x, tok))
                        r.collect(x, tok, &s_count, full);
                }, [](int) {});
                found = r.collected(&s_count);
            }
        }
        if (part != 0) {
            r.leave();
            return;
        }
        const double log_total = log(total);
        const u64 *sorted = r.list;
        if (found <= kThreads) {                          // each to its rank
            const u64 key = tid < found ? r.list[tid] : ~0ull;
            int rank = 0;
            if (warp * 32 < found)
                for (int j = 0; j < found; ++j)
                    rank += r.list[j] < key;
            if (tid < found)
                r.bins[rank] = key;
            sorted = r.bins;
            __syncthreads();
        } else
            sort_list(r.list, found);
        for (int i = tid; i < p.n; i += kThreads) {
            const u64 e = i < found ? sorted[i] : 0;
            const float x = logit_of((unsigned)(e >> 32));
            const double z = x == m ? 0.0 : ((double)x - (double)m) * c * 0.6931471805599453;
            p.ids[(long long)row * p.n + i] = i < found ? (int)(unsigned)e : -1;
            p.logp[(long long)row * p.n + i] = i < found ? (float)(z - log_total) : -CUDART_INF_F;
        }
        r.leave();
        return;
    }

    int token = -1;                                       // in warp 0 of one CTA of the cluster
    u64 mass = 0;
    if (m == -CUDART_INF_F) {
        // nothing above -infinity: the first allowed token that is not NaN, if there is one
        int first = kNone;
        for (int i = r.c0 * p.blocks * kU * 32 * N - r.view.head + tid; i < min(p.V, r.c1 * p.blocks * kU * 32 * N - r.view.head); i += kThreads)
            if (i >= 0 && i < first && r.view.allowed(i) && r.view.one(i) == -CUDART_INF_F)
                first = i;
        first = __reduce_min_sync(kFull, first);
        __syncthreads();
        if (lane == 0)
            reinterpret_cast<int *>(s_scratch)[warp] = first;
        __syncthreads();
        first = __reduce_min_sync(kFull, lane < kWarps ? reinterpret_cast<int *>(s_scratch)[lane] : kNone);
        const Word w = r.exchange({0.0, 0, 0.f, first});
        first = __reduce_min_sync(kFull, lane < size ? w.token : kNone);
        if (tid == 0 && part == 0)
            finish(first == kNone ? -1 : first, -CUDART_INF_F, 0.f);
        r.barrier();
        return;
    }
    const bool greedy = cold || top_k == 1 || !(top_p > 0.f) || min_p > 1.f;
    if (greedy) {
        // the first chunk with the maximum, of the first CTA that has one
        auto best = [m](float x, int) { return (u64)(x == m); };
        for (int i = tid; i < r.c1 - r.c0; i += kThreads)
            r.chunk_mass[i] = r.chunk_max[i] == m ? 1 : 0;
        __syncthreads();
        r.mine = own_max == m ? 1 : 0;
        r.before = __any_sync(kFull, lane < part && all.m == m) ? 1 : 0;
        token = r.find(best, 0);
        if (warp == 0 && lane == 0 && token >= 0)
            finish(token, cold ? 0.f : (float)-log(total), cold ? 1.f : (float)(1.0 / total));
        r.barrier();
        return;
    }
    Cut cut = {-CUDART_INF_F, kNone};
    auto tighten = [&](const Cut &o) {
        if (o.tighter_than(cut))
            cut = o;
    };
    auto kept_weight = [&](float x, int tok) { return cut.keeps(x, tok) ? r.weight(x) : (u64)0; };
    if (plain) {
        for (int i = tid; i < r.c1 - r.c0; i += kThreads)
            r.chunk_mass[i] = r.chunk_max[i] > -CUDART_INF_F ? (u64)__double2ll_rn(chunk_sum(i, m) * r.unit) : 0;
        __syncthreads();
        mass = r.share_masses();
    } else {
        const float low = min_p <= 0.f ? -CUDART_INF_F : m == CUDART_INF_F ? m : fminf(m, __double2float_ru((double)m + log((double)min_p) * (1.4426950408889634 / c)));
        // A list of the tokens that can be kept, where few can
        bool reached = min_p > 0.f;
        int last = min_p > 0.f ? r.bin_of(low) : kBins - 1;
        if (top_k > 0 && top_k <= kList) {
            bool some;
            const int b = r.reach([](float) { return 1u; }, (u64)top_k, some);
            last = min(last, b);
            reached = true;
        } else if (top_k <= 0 && min_p <= 0.f) {
            // the lanes' maxima hold top_p of the whole sum (each counted somewhat too low)
            const float most = 0x1p+31f / (float)(p.per * 32);
            last = r.reach([&](float x) { return (unsigned)(x == m ? most : exp2_fast((x - m) * c32) * 0.9999847f * most); },
                           (u64)((double)top_p * total * (double)most) + 2, reached);
        }
        int found = kList + 1;
        if (reached)
            found = r.gather(last, &s_count, &s_hits);
        else
            r.barrier();                                  // (every CTA's bins have been read)
        if (found <= kList) {
            if (part == 0)
                from_list(r, found, top_k, low, top_p, exact_sum ? (u64)__double2ll_rn(total * r.unit) : 0, u, &s_left,
                          [&](int tok, float x, u64 kept) {
                              const double z = x == m ? 0.0 : ((double)x - (double)m) * c * 0.6931471805599453;
                              finish(tok, (float)(z - log(total)), (float)((double)kept / r.unit / total));
                          });
            r.leave();
            return;
        }
        if (min_p > 0.f)
            tighten({low, kNone});
        if (top_k > 0) {
            Cut k;
            if (r.template select<unsigned>([](float, int) { return 1u; }, (u64)top_k, k))
                tighten(k);
        }
        // (top_p's border lies within what the other cuts keep, or at its end)
        mass = exact_sum ? (u64)__double2ll_rn(total * r.unit) : r.mass_pass(kept_weight);
        if (top_p < 1.f)
            mass = r.cut_mass(total, part_of(mass, top_p, true), &s_count, cut);
    }
    token = r.find(kept_weight, part_of(mass, u, false));
    if (warp == 0 && lane == 0 && token >= 0) {
        const float x = r.view.one(token);
        const double z = x == m ? 0.0 : ((double)x - (double)m) * c * 0.6931471805599453;
        const double sums = plain ? (double)mass / r.unit : total;
        finish(token, (float)(z - log(sums)), plain ? 1.f : (float)((double)mass / r.unit / sums));
    }
    r.barrier();
}

}  // namespace

namespace {

// CTAs of a row of so many blocks, `uneven`: some rows may take several more passes than others - as far as the host
// knows: it sees which settings are given, not what they hold, and where top_k or min_p is given they mostly leave
// rows that can be listed.  (Given with nothing in it, such a setting costs the second of the figures below.)  Three CTAs an SM,
// in shares of at least 8 blocks, up to four where shares are of 128 (512 x 256,000, the 256 most likely: 144 us
// with two CTAs a row, 169 with one, 160 with four; 128 x 128,256 bf16 from the whole distribution: 43 us with
// four, 54 with eight); eight with uneven rows (300 x 128,256 with top_p 0.95: 235 - 268 us with four, 319 - 366 with two).
// Sixteen only where all rows run at once (4 x 256,000 18.6 us, with eight 21.9).
int cluster_size(int rows, int blocks, int sms, bool uneven)
{
    int size = 1;
    while (size < 8 && ((rows * (long long)size < (uneven ? 8 : 3) * sms && blocks >= 16 * size) ||
                        (rows * (long long)size < 4 * sms && blocks >= 256 * size)))
        size *= 2;
    while (size < kMaxCluster && rows * (long long)kMaxCluster <= sms && blocks >= 16 * size)
        size *= 2;
    return size;
}

// Checks and launch shared by both operators; `p` holds what is theirs alone.
template <bool TOP>
int run(const char *name, const cstr_table_t *const *tables, int32_t n_tables, const int32_t *row_table,
        const int32_t *states, const void *logits, int32_t dtype, int64_t ld, int32_t vocab_size, int32_t rows,
        SampleParams &p, cudaStream_t stream)
{
    if ((uintptr_t)logits % (dtype == CSTR_BF16 ? 2 : 4))
        return cstr_fail(CSTR_ERR_SHAPE, "%s: logits must start on whole elements", name);
    int device = -1;
    CSTR_CUDA_TRY(cudaGetDevice(&device));
    if (const int rc = cstr_rows::take_tables(name, tables, n_tables, row_table, states, vocab_size, device, p.t))
        return rc;
    int sms = 0;
    if (const int rc = cstr_rows::sm_count(device, sms))
        return rc;
    p.logits = logits;
    p.ld = ld;
    p.V = vocab_size;
    p.rows = rows;
    p.oob = CSTR_OOB_RECORD();
    const bool bf16 = dtype == CSTR_BF16;
    const int n = bf16 ? 8 : 4;
    const int blocks = (vocab_size + n - 1 + 32 * kU * n - 1) / (32 * kU * n);       // (a row may begin inside a vector)
    const int size = cluster_size(rows, blocks, sms, p.top_p && !p.top_k && !p.min_p);
    if ((long long)rows * size > 0x7fffffffLL)
        return cstr_fail(CSTR_ERR_SHAPE, "%s: rows x vocabulary too large for one launch", name);
    p.blocks = (blocks + kMaxChunks * size - 1) / (kMaxChunks * size);
    const int chunks = (blocks + p.blocks - 1) / p.blocks;
    p.per = (chunks + size - 1) / size;
    p.scale_bits = 62;
    while ((1LL << (62 - p.scale_bits)) < vocab_size)
        --p.scale_bits;
    auto bytes = [](int chunks) { return (2 * kList + chunks) * 8 + chunks * 33 * 4; };
    void (*kernel)(SampleParams) = bf16 ? sample_kernel<true, TOP> : sample_kernel<false, TOP>;
    static cstr_rows::LaunchLimits<2> limits;
    if (const int rc = limits.set(kernel, bf16, device, kMaxCluster, bytes(kMaxChunks)))
        return rc;
    return cstr_launch(kernel, (long long)rows * size, kThreads, size, bytes(p.per), stream, p);
}

int check_rows(const char *name, int32_t n_tables, int32_t dtype, int64_t ld, int32_t vocab_size, int32_t rows)
{
    if (n_tables < 0 || n_tables > CSTR_MAX_TABLES)
        return cstr_fail(CSTR_ERR_ARG, "%s: n_tables = %d, need 0..%d", name, n_tables, CSTR_MAX_TABLES);
    if (dtype != CSTR_F32 && dtype != CSTR_BF16)
        return cstr_fail(CSTR_ERR_DTYPE, "%s: unknown dtype %d", name, dtype);
    if (rows < 0 || vocab_size < 1 || vocab_size > CSTR_MAX_ROW)
        return cstr_fail(CSTR_ERR_ARG, "%s: rows = %d, vocab_size = %d", name, rows, vocab_size);
    if (ld < vocab_size)
        return cstr_fail(CSTR_ERR_SHAPE, "%s: ld = %lld is below V = %d", name, (long long)ld, vocab_size);
    return CSTR_OK;
}

}  // namespace

extern "C" int cstr_sample(const cstr_table_t *const *tables, int32_t n_tables, const int32_t *row_table,
                           const int32_t *states_in, int32_t *states_out, const void *logits, int32_t dtype,
                           int64_t ld, int32_t vocab_size, const float *uniform, const float *temperature,
                           const int32_t *top_k, const float *top_p, const float *min_p, int32_t *tokens_out,
                           float *logp_out, float *kept_out, uint8_t *accept_out, int32_t rows, void *cuda_stream)
{
    if (const int rc = check_rows("cstr_sample", n_tables, dtype, ld, vocab_size, rows))
        return rc;
    if (rows == 0)
        return CSTR_OK;
    if (!logits || !uniform || !tokens_out || (n_tables > 0 && (!tables || !states_in || !states_out)))
        return cstr_fail(CSTR_ERR_NULL, "cstr_sample: null pointer");
    SampleParams p;
    memset(&p, 0, sizeof p);
    p.uniform = uniform;
    p.temperature = temperature;
    p.top_k = top_k;
    p.top_p = top_p;
    p.min_p = min_p;
    p.states_out = n_tables > 0 ? states_out : nullptr;
    p.tokens = tokens_out;
    p.logp = logp_out;
    p.kept = kept_out;
    p.accept_out = accept_out;
    return run<false>("cstr_sample", tables, n_tables, row_table, states_in, logits, dtype, ld, vocab_size, rows, p,
                      (cudaStream_t)cuda_stream);
}

extern "C" int cstr_top_logprobs(const cstr_table_t *const *tables, int32_t n_tables, const int32_t *row_table,
                                 const int32_t *states, const void *logits, int32_t dtype, int64_t ld,
                                 int32_t vocab_size, float temperature, int32_t n, int32_t *ids_out,
                                 float *logp_out, float *lse_out, int32_t rows, void *cuda_stream)
{
    if (const int rc = check_rows("cstr_top_logprobs", n_tables, dtype, ld, vocab_size, rows))
        return rc;
    if (n < 1 || n > CSTR_MAX_TOP)
        return cstr_fail(CSTR_ERR_ARG, "cstr_top_logprobs: n = %d, need 1..%d", n, CSTR_MAX_TOP);
    const double c = 1.4426950408889634 / temperature;
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite((float)c))
        return cstr_fail(CSTR_ERR_ARG, "cstr_top_logprobs: temperature = %g", temperature);
    if (rows == 0)
        return CSTR_OK;
    if (!logits || !ids_out || !logp_out || (n_tables > 0 && (!tables || !states)))
        return cstr_fail(CSTR_ERR_NULL, "cstr_top_logprobs: null pointer");
    SampleParams p;
    memset(&p, 0, sizeof p);
    p.n = n;
    p.c = c;
    p.ids = ids_out;
    p.logp = logp_out;
    p.lse = lse_out;
    return run<true>("cstr_top_logprobs", tables, n_tables, row_table, states, logits, dtype, ld, vocab_size, rows, p,
                     (cudaStream_t)cuda_stream);
}
