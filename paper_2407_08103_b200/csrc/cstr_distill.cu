// Divergence of a student's constrained distribution from a teacher's record of its most likely tokens,
// forward and gradient, in one kernel.
//
// Mathematics, with c = log2(e) / temperature, e_v = 2^(c (x_v - m)): the record's tokens are kept out of the
// running sum of the others, so that what the others hold together is a sum of its own and no small difference
// (the record often holds all but 1e-4).  With t the record, T = sum t, r the rest of the teacher, S = sum e:
//   loss = sum t_i (log t_i - log e_i / S) + r (log r - log rest / S)
//   d loss / d z_v = (T + r) e_v / S - (v in the record: t_v, else r e_v / rest)
// The sums over the record are taken in 64 bits (a divergence is a small difference of them), those over the
// vocabulary in 32.
//
// Bound: logits read once, gradient written once.  A cluster of CTAs shares a row, sized so that there are about as
// many CTAs as the SMs hold (eight of 32 registers each: 2,048 x 32,000 bf16 80 us, 3.3 TB/s, with six 89 us): the
// phases of a row - its record, one pass, the join, the gradient - take as long as their latencies, and other rows
// fill them.  512 x 256,000 fp32 with gradient 270 us, 3.9 TB/s of what has to move (5.8 TB/s of what does: the
// gradient's pass finds half the row in the L2 cache), its loss alone 126 us.  A bitmap in shared memory marks the
// record's tokens of a CTA's share; their gradients are written behind the others'.  Measured and dropped: the
// record left to one warp (512 x 256,000 311 us against 290 then), the row brought to the L2 cache ahead (288), the gradient's pass backwards (279 against 272).
#include <cooperative_groups.h>
#include <math.h>
#include <string.h>

#include "cstr_rows.cuh"

namespace cg = cooperative_groups;

namespace {

using namespace cstr_rows;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;
constexpr int kCtas = 8;                 // of an SM

struct DistillParams {
    Tables t;
    const void *logits;
    void *dlogits;
    long long ld;
    int V, rows, k, tail;
    float c;                         // log2(e) / temperature
    double inv_temp;
    const int32_t *ids;
    const float *teacher, *weight;
    float *loss;
    unsigned words;                  // of a CTA's bitmap
    unsigned long long *oob;
};

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

// A CTA's part of the record.  Weights are relative to exp(ref), logits to x, their largest: t = sum t_i,
// t_log = sum t_i log t_i, t_x = sum t_i (x_i - x), e = sum of the distinct tokens' 2^(c (x_i - x)).
struct Record {
    double t, t_log, t_x, given;
    float ref, x, e;
};
__device__ __forceinline__ Record join(const Record &a, const Record &b, float c)
{
    Record r = {0.0, 0.0, 0.0, a.given + b.given, fmaxf(a.ref, b.ref), fmaxf(a.x, b.x), 0.f};
    auto add = [&](const Record &o) {
        if (o.t == 0.0 && o.e == 0.f)            // (nothing in it; its references are -infinity)
            return;
        const double down = o.ref == r.ref ? 0.0 : (double)o.ref - (double)r.ref, f = down == 0.0 ? 1.0 : exp(down);
        r.t += f * o.t;
        r.t_log += f == 0.0 ? 0.0 : f * (o.t_log + o.t * down);
        r.t_x += f * (o.x == r.x ? o.t_x : o.t_x + o.t * ((double)o.x - (double)r.x));
        r.e += o.x == r.x ? o.e : o.e * exp2_fast((o.x - r.x) * c);
    };
    add(a);
    add(b);
    return r;
}

// What a CTA knows of its share of the row.
struct Share {
    MaxSum rest;
    Record record;
};

template <class T> __device__ __forceinline__ T from_lane(const T &v, int off)
{
    T r;
    const int n = sizeof(T) / 4;
    const int *a = reinterpret_cast<const int *>(&v);
    int *b = reinterpret_cast<int *>(&r);
#pragma unroll
    for (int i = 0; i < n; ++i)
        b[i] = __shfl_xor_sync(kFull, a[i], off);
    return r;
}

template <bool BF16> __device__ __forceinline__ void store_one(char *row, int tok, float x)
{
    if (BF16) {
        unsigned u;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(0.f), "f"(x));
        ((unsigned short *)row)[tok] = (unsigned short)u;
    } else
        ((float *)row)[tok] = x;
}

template <bool BF16> __device__ __forceinline__ uint4 narrow(const float *d)
{
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (BF16)
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(d[BF16 ? 2 * i + 1 : i]), "f"(d[BF16 ? 2 * i : i]));
        else
            w[i] = __float_as_uint(d[i]);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// x = 2^(c (x - ref)), two logits per instruction but for the exponential itself
template <int CNT> __device__ __forceinline__ void exponentials(float (&x)[CNT], float ref, float c)
{
#pragma unroll
    for (int i = 0; i < CNT; i += 2) {
        asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %2};\nadd.rn.f32x2 a, a, b;\n"
            "mov.b64 b, {%3, %3};\nmul.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}\n"
            : "+f"(x[i]), "+f"(x[i + 1]) : "f"(-ref), "f"(c));
        x[i] = exp2_fast(x[i]);
        x[i + 1] = exp2_fast(x[i + 1]);
    }
}

// WIDE: rows of both buffers begin at the same place of their 16 bytes (or there is no gradient).
// kUnroll: vectors of a thread in flight.
template <bool BF16, bool WIDE, int kUnroll>
__global__ void __launch_bounds__(kThreads, kCtas)
distill_kernel(const __grid_constant__ DistillParams p)
{
    using View = RowView<BF16>;
    constexpr int N = View::N;
    extern __shared__ unsigned s_dynamic[];              // bitmap, then ids, weights and logits of the record
    __shared__ Share s_warp[kWarps], s_share, s_sums;    // the warps', the CTA's, the row's
    __shared__ MaxSum s_all;
    __shared__ float s_top[2][kWarps];                   // largest teacher value, largest logit of the record's part
    __shared__ float s_result[5];                        // factors of e in the rest, in the record, of t; maxima
    __shared__ float s_ref;
    __shared__ int s_twice, s_count[kWarps];
    unsigned *bitmap = s_dynamic;
    int *s_id = reinterpret_cast<int *>(bitmap + p.words);
    float *s_t = reinterpret_cast<float *>(s_id + p.k), *s_x = s_t + p.k;
    cstr_wait_for_earlier_kernels();
    cstr_let_next_kernel_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int size = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / size;
    int table, state;
    const uint32_t *mrow;
    const bool active = row_state(p.t, row, table, state, mrow);
    const float w = p.weight ? p.weight[row] : 1.f;
    const View view(p.logits, (long long)row * p.ld, p.V, mrow);
    char *d_row = (char *)p.dlogits + (long long)row * p.ld * View::ESZ;
    const int vectors = view.vectors(), per = (vectors + size - 1) / size;
    const int v0 = min(part * per, vectors), v1 = min(v0 + per, vectors);
    // the share's vectors that are inside the row; the row's first and last one may be not
    const int i0 = v0 + (v0 == 0 && view.head > 0 ? 1 : 0), i1 = v1 - (v1 == vectors && i0 < v1 && !view.inside(vectors - 1) ? 1 : 0);
    const int edge = tid == 0 && v0 < i0 ? v0 : tid == 32 && i1 < v1 ? i1 : -1;      // ... by one thread each
    const uint4 *x_vec = reinterpret_cast<const uint4 *>(view.row - view.head * View::ESZ);
    uint4 *d_vec = reinterpret_cast<uint4 *>(d_row - view.head * View::ESZ);
    auto put_one = [&](int v, const float (&d)[N]) {
        for (int e = 0; e < N; ++e)
            if (view.token(v) + e >= 0 && view.token(v) + e < p.V)
                store_one<BF16>(d_row, view.token(v) + e, d[e]);
    };
    auto put = [&](int v, const float (&d)[N]) {
        if (WIDE)
            __stcs(d_vec + v, narrow<BF16>(d));
        else
            put_one(v, d);
    };
    if (!active || w == 0.f) {
        const float zero[N] = {};
        if (p.dlogits) {
            for (int v = i0 + tid; v < i1; v += kThreads)
                put(v, zero);
            if (edge >= 0)
                put_one(edge, zero);
        }
        if (part == 0 && tid == 0)
            p.loss[row] = 0.f;
        return;
    }

    // the record's tokens of this share, in the record's order
    const int lo = max(view.token(v0), 0), hi = min(view.token(v1), p.V), base = view.token(v0);
    const int32_t *ids = p.ids + (long long)row * p.k;
    const float *teacher = p.teacher + (long long)row * p.k;
    for (int i = tid; i < (int)p.words; i += kThreads)
        bitmap[i] = 0;
    if (tid == 0)
        s_twice = 0;
    int mine = 0;                                        // entries of this share
    for (int k0 = 0; k0 < p.k; k0 += kThreads) {
        const int i = k0 + tid, id = i < p.k ? ids[i] : -1;
        const float g = i < p.k ? teacher[i] : 0.f;
        const bool in = id >= lo && id < hi && g != -CUDART_INF_F;
        const unsigned who = __ballot_sync(kFull, in);
        if (lane == 0)
            s_count[warp] = __popc(who);
        __syncthreads();
        int at = mine + __popc(who & ((1u << lane) - 1));
#pragma unroll
        for (int j = 0; j < kWarps; ++j) {
            at += j < warp ? s_count[j] : 0;
            mine += s_count[j];
        }
        if (in) {
            s_id[at] = id;
            s_t[at] = g;
            const unsigned bit = 1u << ((id - base) & 31);
            if (CSTR_INB(p.oob, (id - base) >> 5, p.words, CSTR_SITE_DISTILL) && (atomicOr(bitmap + ((id - base) >> 5), bit) & bit))
                s_twice = 1;
        }
        __syncthreads();
    }
    // the first entry's logit comes while the others are read
    const int id_0 = tid < mine ? s_id[tid] : -1;
    const float x_0 = id_0 >= 0 && view.allowed(id_0) ? view.one(id_0) : -CUDART_INF_F;

    // All tokens; with a lumped tail those outside the record.
    const bool lump = p.tail == CSTR_TAIL_LUMP, renorm = p.tail == CSTR_TAIL_RENORM;
    auto others = [&](int v) {
        const int bit = (v - v0) * N;
        return lump ? ~(bitmap[bit >> 5] >> (bit & 31)) : kFull;
    };
    // A likely token's sum swallows the last bits of hundreds of unlikely ones, all to the same side: what was added
    // too much is kept along (log q of 512 x 256,000: root mean square error 1.0e-6 without).
    MaxSum rest = {-CUDART_INF_F, 0.f};
    float over = 0.f;
    auto add = [&](uint4 raw) {
        float x[N], top = -CUDART_INF_F;
#pragma unroll
        for (int e = 0; e < N; ++e)
            x[e] = View::plain(raw, e);
#pragma unroll
        for (int e = 0; e < N; e += 2)
            top = max3(top, x[e], x[e + 1]);
        if (top > rest.m) {
            const float f = exp2_fast((rest.m - top) * p.c);
            rest.s *= f;
            over *= f;
            rest.m = top;
        }
        exponentials(x, rest.m == -CUDART_INF_F ? 0.f : rest.m, p.c);
        float s[2] = {x[0], x[1]};
#pragma unroll
        for (int e = 2; e < N; ++e)
            s[e & 1] += x[e];
        const float y = s[0] + s[1] - over, sum = rest.s + y;
        over = sum - rest.s - y;
        rest.s = sum;
    };
#pragma unroll 1
    for (int v = i0 + tid; v < i1; v += kUnroll * kThreads) {
        uint4 raw[kUnroll];
        unsigned bits[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            bits[u] = 0u;
            raw[u] = make_uint4(0u, 0u, 0u, 0u);
            if (v + u * kThreads < i1) {
                raw[u] = x_vec[v + u * kThreads];
                bits[u] = view.bits(v + u * kThreads) & others(v + u * kThreads);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            add(View::mask(raw[u], bits[u]));
    }
    if (edge >= 0)
        add(View::mask(view.edge(edge), others(edge)));
    rest.s -= over;

    // the record's part: largest teacher value and logit, then the sums relative to them (by the warps that
    // have entries)
    const bool any = warp * 32 < mine;
    Record rec = {0.0, 0.0, 0.0, 0.0, -CUDART_INF_F, -CUDART_INF_F, 0.f};
    if (any) {
        for (int i = tid; i < mine; i += kThreads) {
            const int id = s_id[i];
            const float x = i == tid ? x_0 : view.allowed(id) ? view.one(id) : -CUDART_INF_F, g = s_t[i];
            s_x[i] = x;
            if (lump)
                rec.given += exp((double)g);
            if (x != -CUDART_INF_F) {
                rec.ref = fmaxf(rec.ref, g);
                rec.x = fmaxf(rec.x, x);
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            rec.ref = fmaxf(rec.ref, __shfl_xor_sync(kFull, rec.ref, off));
            rec.x = fmaxf(rec.x, __shfl_xor_sync(kFull, rec.x, off));
        }
    }
    if (lane == 0) {
        s_top[0][warp] = rec.ref;
        s_top[1][warp] = rec.x;
    }
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) {
        rec.ref = fmaxf(rec.ref, s_top[0][i]);
        rec.x = fmaxf(rec.x, s_top[1][i]);
    }
    if (!renorm)
        rec.ref = 0.f;
    const bool twice = s_twice != 0;
    // an id's first entry in the record
    auto first = [&](int i) {
        if (twice)
            for (int j = 0; j < i; ++j)
                if (s_id[j] == s_id[i])
                    return false;
        return true;
    };
    if (any) {
        for (int i = tid; i < mine; i += kThreads) {
            if (s_x[i] == -CUDART_INF_F)
                continue;
            const double log_t = (double)s_t[i] - (double)rec.ref, t = exp(log_t);
            rec.t += t;
            rec.t_log += t == 0.0 ? 0.0 : t * log_t;
            rec.t_x += t * ((double)s_x[i] - (double)rec.x);
            if (lump && first(i))
                rec.e += exp2_fast((s_x[i] - rec.x) * p.c);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            rec.t += __shfl_xor_sync(kFull, rec.t, off);
            rec.t_log += __shfl_xor_sync(kFull, rec.t_log, off);
            rec.t_x += __shfl_xor_sync(kFull, rec.t_x, off);
            rec.given += __shfl_xor_sync(kFull, rec.given, off);
            rec.e += __shfl_xor_sync(kFull, rec.e, off);
        }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        rest = join(rest, from_lane(rest, off), p.c);
    if (lane == 0)
        s_warp[warp] = {rest, rec};
    __syncthreads();
    if (warp == 0) {
        // (all with the same references)
        Share s = s_warp[lane & (kWarps - 1)];
#pragma unroll
        for (int off = kWarps / 2; off > 0; off >>= 1)
            s.rest = join(s.rest, from_lane(s.rest, off), p.c);
        for (int i = 1; i * 32 < mine && i < kWarps; ++i) {
            s.record.t += lane == 0 ? s_warp[i].record.t : 0.0;
            s.record.t_log += lane == 0 ? s_warp[i].record.t_log : 0.0;
            s.record.t_x += lane == 0 ? s_warp[i].record.t_x : 0.0;
            s.record.given += lane == 0 ? s_warp[i].record.given : 0.0;
            s.record.e += lane == 0 ? s_warp[i].record.e : 0.f;
        }
        if (lane == 0)
            s_share = s;
        __syncwarp();
    }
    if (size > 1)
        cluster.sync();
    auto teachers_rest = [](const Share &s) {
        const double left = 1.0 - s.record.given;
        return left < 0.0 ? 0.0 : left;
    };
    if (warp == 0) {
        Share s = {{-CUDART_INF_F, 0.f}, {0.0, 0.0, 0.0, 0.0, -CUDART_INF_F, -CUDART_INF_F, 0.f}};
        if (lane < size)
            s = *cluster.map_shared_rank(&s_share, lane);
        for (int off = size / 2; off > 0; off >>= 1) {
            s.rest = join(s.rest, from_lane(s.rest, off), p.c);
            s.record = join(s.record, from_lane(s.record, off), p.c);
        }
        if (lane == 0) {
            const MaxSum all = lump ? join(s.rest, {s.record.x, s.record.e}, p.c) : s.rest;
            if (s.record.ref == CUDART_INF_F)
                s.record.t = CUDART_NAN;         // a record with infinite logits is none
            s_sums = s;
            s_all = all;
            float f_rest = 0.f, f_listed = 0.f, f_t = 0.f;
            if (all.m != -CUDART_INF_F || all.s != 0.f) {
                const float t = (float)s.record.t, wt = (float)((double)w * p.inv_temp);
                float sum = renorm ? (t != 0.f ? t / t : 0.f) : t;
                if (lump && s.rest.s != 0.f) {
                    // the rest's tokens are counted from their own maximum: they may lie far below the record's
                    const float left = (float)teachers_rest(s);
                    sum += left;
                    f_rest = wt * (sum * exp2_fast((s.rest.m - all.m) * p.c) / all.s - left / s.rest.s);
                }
                f_listed = wt * sum / all.s;
                if (!lump)
                    f_rest = f_listed;
                f_t = renorm ? (t != 0.f ? wt / t : 0.f) : wt;
            }
            s_result[0] = f_rest;
            s_result[1] = f_listed;
            s_result[2] = f_t;
            s_result[3] = all.m;
            s_result[4] = s.rest.m;
            s_ref = s.record.ref;
        }
    }
    if (size > 1) {                              // the shares have been read; the end waits for that
        __syncwarp();
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    }
    // The row's loss, by one thread: behind the gradient, which does not wait for it.
    auto write_loss = [&]() {
        const Share sums = s_sums;
        const MaxSum all = s_all;
        const Record &r = sums.record;
        float loss = 0.f;
        if (all.m != -CUDART_INF_F || all.s != 0.f) {
            // log S relative to the record's largest logit
            const double inv = p.inv_temp, total = all.s;
            const double log_all = log(total) + (r.x == all.m ? 0.0 : ((double)all.m - (double)r.x) * inv);
            double value = r.t == 0.0 ? 0.0 : r.t_log - r.t_x * inv + r.t * log_all;
            if (renorm)
                value = r.t != 0.0 ? value / r.t - log(r.t) : 0.0;
            const double left = lump && sums.rest.s != 0.f ? teachers_rest(sums) : 0.0;
            if (left != 0.0)
                value += left * (log(left / ((double)sums.rest.s / total)) - (sums.rest.m == all.m ? 0.0 : ((double)sums.rest.m - (double)all.m) * inv));
            loss = (float)((double)w * value);
        }
        p.loss[row] = loss;
    };
    if (!p.dlogits) {
        if (part == 0 && tid == 0)
            write_loss();
        if (size > 1)
            asm volatile("barrier.cluster.wait;" ::: "memory");
        return;
    }
    __syncthreads();
    const float f_rest = s_result[0], low = s_result[4];
    // A token that is left out is -infinity here: its exponential and with it its gradient are 0 - unless the
    // factor or the maximum is not finite.
    const bool plain = fabsf(f_rest) < CUDART_INF_F && fabsf(low) < CUDART_INF_F;
    auto slope = [&](uint4 raw, float (&d)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            d[e] = View::plain(raw, e);
        if (plain) {
            exponentials(d, low, p.c);
#pragma unroll
            for (int e = 0; e < N; ++e)
                d[e] *= f_rest;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                d[e] = d[e] == -CUDART_INF_F ? 0.f : f_rest * exp2_fast((d[e] - low) * p.c);
        }
    };
#pragma unroll 1
    for (int v = i0 + tid; v < i1; v += kUnroll * kThreads) {
        uint4 raw[kUnroll];
        unsigned bits[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            bits[u] = 0u;
            raw[u] = make_uint4(0u, 0u, 0u, 0u);
            if (v + u * kThreads < i1) {
                raw[u] = __ldcs(x_vec + v + u * kThreads);
                bits[u] = view.bits(v + u * kThreads) & others(v + u * kThreads);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float d[N];
            slope(View::mask(raw[u], bits[u]), d);
            if (v + u * kThreads < i1)
                put(v + u * kThreads, d);
        }
    }
    if (edge >= 0) {
        float d[N];
        slope(View::mask(view.edge(edge), others(edge)), d);
        put_one(edge, d);
    }
    __syncthreads();                             // the record's tokens behind what has been written in their places
    const float f_listed = s_result[1], f_t = s_result[2], ref = s_result[3];
    const double t_ref = s_ref;                  // 0 unless the record is renormalised
    for (int i = tid; i < mine; i += kThreads) {
        if (!first(i) || !CSTR_INB(p.oob, s_id[i], p.V, CSTR_SITE_DISTILL))
            continue;
        float d = 0.f;
        if (s_x[i] != -CUDART_INF_F) {
            double t = 0.0;
            for (int j = i; j < (twice ? mine : i + 1); ++j)
                if (s_id[j] == s_id[i])
                    t += exp((double)s_t[j] - t_ref);
            d = f_listed * exp2_fast((s_x[i] - ref) * p.c) - (float)(t * (double)f_t);
        }
        store_one<BF16>(d_row, s_id[i], d);
    }
    if (part == 0 && tid == kThreads - 1)
        write_loss();
    if (size > 1)
        asm volatile("barrier.cluster.wait;" ::: "memory");
}

}  // namespace

extern "C" int cstr_distill_loss(const cstr_table_t *const *tables, int32_t n_tables, const int32_t *row_table,
                                 const int32_t *states, const void *logits, int32_t dtype, int64_t ld,
                                 int32_t vocab_size, float temperature, const int32_t *teacher_ids,
                                 const float *teacher_logp, int32_t k, int32_t tail, const float *weight,
                                 float *loss_out, void *dlogits, int32_t rows, void *cuda_stream)
{
    if (n_tables < 0 || n_tables > CSTR_MAX_TABLES)
        return cstr_fail(CSTR_ERR_ARG, "cstr_distill_loss: n_tables = %d, need 0..%d", n_tables, CSTR_MAX_TABLES);
    if (dtype != CSTR_F32 && dtype != CSTR_BF16)
        return cstr_fail(CSTR_ERR_DTYPE, "cstr_distill_loss: unknown dtype %d", dtype);
    if (rows < 0 || vocab_size < 1 || vocab_size > CSTR_MAX_ROW)
        return cstr_fail(CSTR_ERR_ARG, "cstr_distill_loss: rows = %d, vocab_size = %d", rows, vocab_size);
    if (k < 1 || k > CSTR_MAX_TOP)
        return cstr_fail(CSTR_ERR_ARG, "cstr_distill_loss: k = %d, need 1..%d", k, CSTR_MAX_TOP);
    if (tail != CSTR_TAIL_DROP && tail != CSTR_TAIL_RENORM && tail != CSTR_TAIL_LUMP)
        return cstr_fail(CSTR_ERR_ARG, "cstr_distill_loss: unknown tail %d", tail);
    const float c = (float)(1.4426950408889634 / temperature);
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(c))
        return cstr_fail(CSTR_ERR_ARG, "cstr_distill_loss: temperature = %g", temperature);
    if (ld < vocab_size)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_distill_loss: ld = %lld is below V = %d", (long long)ld, vocab_size);
    if (rows == 0)
        return CSTR_OK;
    if (!logits || !teacher_ids || !teacher_logp || !loss_out || (n_tables > 0 && (!tables || !states)))
        return cstr_fail(CSTR_ERR_NULL, "cstr_distill_loss: null pointer");
    const bool bf16 = dtype == CSTR_BF16;
    const uintptr_t element = bf16 ? 2 : 4;
    if ((uintptr_t)logits % element || (uintptr_t)dlogits % element)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_distill_loss: logits and dlogits must start on whole elements");
    int device = -1;
    CSTR_CUDA_TRY(cudaGetDevice(&device));
    DistillParams p;
    memset(&p, 0, sizeof p);
    if (const int rc = cstr_rows::take_tables("cstr_distill_loss", tables, n_tables, row_table, states, vocab_size, device, p.t))
        return rc;
    p.logits = logits;
    p.dlogits = dlogits;
    p.ld = ld;
    p.V = vocab_size;
    p.rows = rows;
    p.k = k;
    p.tail = tail;
    p.c = c;
    p.inv_temp = 1.0 / (double)temperature;
    p.ids = teacher_ids;
    p.teacher = teacher_logp;
    p.weight = weight;
    p.loss = loss_out;
    p.oob = CSTR_OOB_RECORD();
    int sms = 0;
    if (const int rc = cstr_rows::sm_count(device, sms))
        return rc;
    // As many CTAs as the SMs hold, three quarters of that with a gradient, while shares have 4,096 tokens or more.
    // (512 x 256,000 fp32 with gradient: 273 us with two CTAs a row, 290 with 16, whose shares would still be in the
    // L2 cache when the gradient is written, 420 with one; without one 126 us with four, 156 with two.)
    // Bitmaps of at most 32 KB (with 16 CTAs 64 KB).
    int size = 1;
    while (size < kMaxCluster && (vocab_size > 262144LL * size ||
                                  (rows * (long long)size < (dlogits ? 6 : 8) * sms && vocab_size >= 8192LL * size)))
        size *= 2;
    if ((long long)rows * size > 0x7fffffffLL)
        return cstr_fail(CSTR_ERR_SHAPE, "cstr_distill_loss: rows x vocabulary too large for one launch");
    const int n = bf16 ? 8 : 4;
    const int vectors = (vocab_size + 2 * n - 2) / n, per = (vectors + size - 1) / size;   // (a row may begin inside a vector)
    p.words = (unsigned)((per * (long long)n + 31) / 32);
    const int smem = (int)p.words * 4 + k * 12;
    const bool together = !dlogits || (((uintptr_t)logits ^ (uintptr_t)dlogits) & 15u) == 0;
    void (*kernel)(DistillParams);
    const int kind = (!together ? 0 : dlogits ? 2 : 4) + bf16;
    if (!together)
        kernel = bf16 ? distill_kernel<true, false, 1> : distill_kernel<false, false, 1>;
    else if (dlogits)
        kernel = bf16 ? distill_kernel<true, true, 1> : distill_kernel<false, true, 1>;
    else
        kernel = bf16 ? distill_kernel<true, true, 2> : distill_kernel<false, true, 2>;
    static cstr_rows::LaunchLimits<6> limits;
    if (const int rc = limits.set(kernel, kind, device, kMaxCluster, (CSTR_MAX_ROW / kMaxCluster / 32 + 2) * 4 + CSTR_MAX_TOP * 12))
        return rc;
    return cstr_launch(kernel, (long long)rows * size, kThreads, size, smem, (cudaStream_t)cuda_stream, p);
}
