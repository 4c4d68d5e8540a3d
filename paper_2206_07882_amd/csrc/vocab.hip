// Beam selection over large vocabularies, from logits: log-softmax, scores and the best extensions of a beam (Sec. 2: up
// to W hypotheses are kept per iteration) in one pass over the logits.
//
// Short rows (a wave holds one in its registers): one launch, one workgroup per utterance.  Long rows, or wide beams of few utterances: a hypothesis'
// candidates are ordered as its logits are, so a stretch of a row can give up all but its n_out largest logits before the
// row's log-sum-exp is known.  First launch: one workgroup per stretch holds it in registers, finds its maximum, sum of
// exponentials and n_out largest logits.  Second launch: one workgroup per utterance joins sums and lists.
//
// The n_out best of many: the n_out-th largest of the best ones of 256 groups bounds the n_out-th best from below; what is not
// below it (few more than n_out) is gathered in LDS and ranked by counting.  Where very many are equal, rank by rank.
#include <float.h>

#include "elem.h"
#include "kernels.h"
#include "select.h"

namespace {

constexpr int MAX_OUT = 64;      // ranks
constexpr int LIST = 512;        // candidates that a selection holds in LDS (more: it goes rank by rank)

struct QrPartHead {
    float top, pad;              // the stretch's largest logit (-inf: none)
    double sum;                  // sum of exp(logit - top); NaN where a logit is NaN or +inf
};

struct QrSelectArgs {
    const float *score;
    const void *logits;
    int64_t ld;
    const uint8_t *finished;
    int log_softmax, end_token;
    int B, W, V, K;
    int n_parts, part;           // stretches of a row, and their length
    int32_t *parent_out, *token_out;
    float *score_out;
    uint8_t *finished_out;
    QrPartHead *heads;           // [B*W][n_parts]
    QrCand *cands;               // [B*W][n_parts][K]: (key of the logit, token), best first, 0: none
};

__device__ __forceinline__ bool is_finished(const QrSelectArgs &a, int64_t row) { return a.finished && a.finished[row]; }
__device__ __forceinline__ bool reads_logits(const QrSelectArgs &a, int64_t row) { return a.score[row] > -INFINITY && !is_finished(a, row); }

// A bound from below of the K-th largest of 256 groups' keys, four to a lane: the K-th largest itself, or a little less (as soon as
// no more than `enough` groups pass); 0 if fewer than K groups have one.  top: the largest.  By bits of the distance from it, which
// begin where the groups' distances do: the first bits of the keys themselves tell little apart.
__device__ __forceinline__ unsigned bound_of(const unsigned (&g)[4], unsigned top, int K, int enough)
{
    unsigned d[4], far = 0u;
    int some = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        d[i] = g[i] ? top - g[i] : ~0u;
        far = g[i] && d[i] > far ? d[i] : far;
        some += (int)__popcll(__ballot(g[i] != 0u));
    }
    if (some < K) return 0u;   // uniform
    far = qr_wave_reduce_u32<true>(far);
    const int bits = 32 - __builtin_clz(far | 1u);
    unsigned D = bits == 32 ? ~0u - 1u : (1u << bits) - 1u;
    for (int bit = bits - 1; bit >= 0; --bit) {
        const unsigned trial = D & ~(1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += (int)__popcll(__ballot(d[i] <= trial));
        if (n >= K) {
            D = trial;   // uniform
            if (n <= enough) break;
        }
    }
    return D < top ? top - D : 1u;
}

// A value as a word: larger double <=> larger word; 0 for what is never taken.
typedef unsigned long long QrValue;
__device__ __forceinline__ QrValue value_word(double v)
{
    if (!(v > -INFINITY)) return 0ull;
    const QrValue u = (QrValue)__double_as_longlong(v + 0.0);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double word_value(QrValue o)
{
    return __longlong_as_double((long long)((o >> 63) ? (o & 0x7FFFFFFFFFFFFFFFull) : ~o));
}
// A candidate of a beam: value, hypothesis, (logit, token).  Better: larger value, then lower hypothesis, then larger logit, then
// lower token.
struct QrPick {
    QrValue v;
    QrCand c;
    int w;
};
__device__ __forceinline__ bool better(const QrPick &p, const QrPick &q) { return p.v != q.v ? p.v > q.v : (p.w != q.w ? p.w < q.w : p.c > q.c); }

struct QrPickList {
    QrValue v[LIST];
    QrCand c[LIST];
    int w[LIST];
    int n;
    QrPick wave_best[16];
};
__device__ __forceinline__ void push(QrPickList &l, const QrPick &p)
{
    const int at = atomicAdd(&l.n, 1);
    if (at < LIST) {
        l.v[at] = p.v;
        l.c[at] = p.c;
        l.w[at] = p.w;
    }
}

__device__ __forceinline__ void put(const QrSelectArgs &a, int b, int r, const QrPick &p)
{
    const int64_t at = (int64_t)b * a.K + r;
    a.parent_out[at] = p.v ? p.w : -1;
    a.token_out[at] = p.v ? qr_cand_index(p.c) : -1;
    a.score_out[at] = p.v ? (float)word_value(p.v) : -INFINITY;
    if (a.finished_out) a.finished_out[at] = p.v && (is_finished(a, (int64_t)b * a.W + p.w) || qr_cand_index(p.c) == a.end_token) ? 1 : 0;
}

// Writes the utterance's ranks from the list, four threads counting for one candidate; each(visit) visits all candidates and is
// what is gone by where the list did not hold them.
template <int THREADS, class Each>
__device__ __forceinline__ void write_ranks(const QrSelectArgs &a, int b, QrPickList &l, Each &&each)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, M = l.n;
    if (M <= LIST) {
        for (int i0 = 0; i0 < M; i0 += THREADS / 4) {   // uniform
            const int i = i0 + (tid >> 2);
            const QrPick mine = {l.v[i < M ? i : 0], l.c[i < M ? i : 0], l.w[i < M ? i : 0]};
            int rank = 0;
            for (int j = tid & 3; j < M; j += 4) rank += better({l.v[j], l.c[j], l.w[j]}, mine) ? 1 : 0;
            rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, true);
            rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, true);
            if ((tid & 3) == 0 && i < M && rank < a.K) put(a, b, rank, mine);
        }
        for (int r = M + tid; r < a.K; r += THREADS) put(a, b, r, {0ull, 0ull, 0});
        return;
    }
    QrPick last = {~0ull, ~0ull, -1};
    for (int r = 0; r < a.K; ++r) {
        QrPick best = {0ull, 0ull, 0x7fffffff};
        each([&](const QrPick &p) {
            if (better(last, p) && better(p, best)) best = p;
        });
        for (int off = 32; off > 0; off >>= 1) {
            const QrPick o = {(QrValue)__shfl_xor(best.v, off), (QrCand)__shfl_xor(best.c, off), __shfl_xor(best.w, off)};
            if (better(o, best)) best = o;
        }
        if (lane == 0) l.wave_best[wave] = best;
        __syncthreads();
        for (int i = 0; i < THREADS / 64; ++i)
            if (better(l.wave_best[i], best)) best = l.wave_best[i];
        __syncthreads();
        if (tid == 0) put(a, b, r, best);
        last = best;
    }
}

// A thread's NV vectors of n logits: vector v of thread t of `threads` starts at element (v * threads + t) * V, wherever the row begins
// in memory (sums have to come out the same for the same row); -inf behind the end.
template <class T, int NV>
struct QrLogits {
    static constexpr int V = QrVec<T>::N, PER = NV * V, GROUP = 8, NG = PER / GROUP;
    static_assert(PER % GROUP == 0, "whole groups");
    float f[PER];
    float best[NG];   // largest of 8 (NaN is passed over)
    __device__ __forceinline__ void load(const T *x, int n, int t, int threads)
    {
        typename QrVec<T>::type raw[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * threads + t) * V;
            if (c + V <= n) {
                raw[v] = *(const typename QrVec<T>::any *)(x + c);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) raw[v][i] = c + i < n ? x[c + i] : (T)-INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) f[i] = (float)raw[i / V][i % V];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            best[g] = -INFINITY;
#pragma unroll
            for (int i = 0; i < GROUP; ++i) best[g] = fmaxf(best[g], f[g * GROUP + i]);
        }
    }
    __device__ __forceinline__ float largest() const
    {
        float m = best[0];
#pragma unroll
        for (int g = 1; g < NG; ++g) m = fmaxf(m, best[g]);
        return m;
    }
    // Relative error at most (16 + 1.2 ln V + 1) 2^-23: 32 additions in fp32; d = top - f and d log2 e are rounded, which weighs d exp(-d), on
    // average ln V at most; a step of exp2.  (fp64 beyond a thread; stretches are joined with one more exponential each.)
    __device__ __forceinline__ float sum_exp(float top) const
    {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) s += qr_exp(f[i] - top);
        return s;
    }
    // take(logit, i) for those that are not below `least`.  A group that has any most often has one, its largest: that one is found
    // without a branch for each.
    template <class Take>
    __device__ __forceinline__ void hits(float least, Take &&take) const
    {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            if (!(best[g] >= least)) continue;
            int n = 0, at = 0;
#pragma unroll
            for (int i = g * GROUP; i < (g + 1) * GROUP; ++i) {
                const bool hit = f[i] >= least;
                n += hit ? 1 : 0;
                at = hit ? i : at;
            }
            if (n == 1) {
                take(best[g], at);
            } else {
#pragma unroll
                for (int i = g * GROUP; i < (g + 1) * GROUP; ++i)
                    if (f[i] >= least) take(f[i], i);
            }
        }
    }
};
__device__ __forceinline__ unsigned logit_key(float f) { return f > -INFINITY ? qr_float_key(f + 0.0f) : 0u; }   // (0 for NaN, too)
// Sum over the wave, on the DPP path (row scans, then the two cross-row broadcasts of gfx9), in all lanes.
__device__ __forceinline__ double wave_sum(double d)
{
#define QR_DPP_ADD(ctrl, rmask)                                                                                          \
    {                                                                                                                    \
        const unsigned long long u = (unsigned long long)__double_as_longlong(d);                                        \
        const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, ctrl, rmask, 0xf, false);          \
        const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), ctrl, rmask, 0xf, false);  \
        d += __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));                                       \
    }
    QR_DPP_ADD(0x111, 0xf)   // row_shr:1
    QR_DPP_ADD(0x112, 0xf)   // row_shr:2
    QR_DPP_ADD(0x114, 0xf)   // row_shr:4
    QR_DPP_ADD(0x118, 0xf)   // row_shr:8
    QR_DPP_ADD(0x142, 0xa)   // row_bcast:15 into rows 1 and 3
    QR_DPP_ADD(0x143, 0xc)   // row_bcast:31 into rows 2 and 3
#undef QR_DPP_ADD
    const unsigned long long u = (unsigned long long)__double_as_longlong(d);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, 63), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), 63);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
// Largest of four neighbouring lanes.
__device__ __forceinline__ unsigned quad_max(unsigned v)
{
    unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true);
    v = o > v ? o : v;
    o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true);
    return o > v ? o : v;
}

// Long rows, first launch.  Grid: x = stretch, y (and z) = row; NT = 256 or 512 threads with NV vectors each.
// Bound by the chain of its steps: of a workgroup's 8 us for 64 x 16 x 32000 bf16 logits (two workgroups one after the other at each
// place, 18 us in all, the second launch 6; vector units busy 41 % or a little more) loading takes 2 to 5, maximum, sums, bound and
// ranks 1 each, gathering 1.6.  Other numbers of waves and logits to one change little, fetching a next stretch ahead spills.
template <class T, int NV, int NT>
__global__ __launch_bounds__(NT, 8) void select_parts_kernel(const QrSelectArgs a)
{
    constexpr int V = QrVec<T>::N, NW = NT / 64;
    __shared__ QrCand list[LIST], wave_best[NW];
    __shared__ unsigned group_best[256];
    __shared__ double sums[NW];
    __shared__ int n_list;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= (int64_t)a.B * a.W || !reads_logits(a, row)) return;   // uniform; the second launch does not ask for it either
    const int first = blockIdx.x * a.part, n = a.V - first < a.part ? a.V - first : a.part;
    if (tid == 0) n_list = 0;
    QrLogits<T, NV> f;
    const T *x = (const T *)a.logits + row * a.ld + first;
    f.load(x, n, tid, NT);
    const float largest = f.largest();   // (NaN is found in the sum)
    if (NT == 256) {
        group_best[tid] = logit_key(largest);
    } else {
        const unsigned k = logit_key(largest), o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)k, 0xB1, 0xf, 0xf, true);   // its neighbour's
        if ((tid & 1) == 0) group_best[tid >> 1] = o > k ? o : k;
    }
    __syncthreads();
    unsigned g[4], top_key = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = group_best[i * 64 + lane];
        top_key = g[i] > top_key ? g[i] : top_key;
    }
    top_key = qr_wave_reduce_u32<true>(top_key);
    const float top = top_key ? qr_key_float(top_key) : -INFINITY;
    if (a.log_softmax) {
        const double d = wave_sum((double)f.sum_exp(top_key ? top : 0.0f));
        if (lane == 0) sums[wave] = d;
    }
    const unsigned T_key = bound_of(g, top_key, a.K, a.K + a.K / 4);
    const float least = T_key > 0x00800000u ? qr_key_float(T_key) : -FLT_MAX;   // (keys up to there are those of -inf and below)
    auto cand = [&](float l, int i) { return qr_cand(qr_float_key(l + 0.0f), first + ((i / V) * NT + tid) * V + i % V); };
    f.hits(least, [&](float l, int i) {
        const int at = atomicAdd(&n_list, 1);
        if (at < LIST) list[at] = cand(l, i);
    });
    __syncthreads();
    const int M = n_list;
    const int64_t part = row * a.n_parts + blockIdx.x;
    QrCand *out = a.cands + part * a.K;
    if (tid == 0) {
        double sum = 0.0;
        if (a.log_softmax)
            for (int w = 0; w < NW; ++w) sum += sums[w];
        a.heads[part] = {top, 0.0f, sum};
    }
    if (M <= LIST) {   // a candidate's rank is how many are better, four threads counting for each
        for (int i0 = 0; i0 < M; i0 += NT / 4) {   // uniform
            const int i = i0 + (tid >> 2);
            const QrCand mine = list[i < M ? i : 0];
            int rank = 0;
#pragma unroll 4
            for (int j = tid & 3; j < M; j += 4) rank += list[j] > mine ? 1 : 0;
            rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, true);
            rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, true);
            if ((tid & 3) == 0 && i < M && rank < a.K) out[rank] = mine;
        }
        if (tid >= M && tid < a.K) out[tid] = 0ull;
        return;
    }
    // many equal logits: rank by rank, from memory (kept in registers up to here they would spill in every call: 26 MB written
    // for 64 x 16 x 32000 bf16, 28 us against 25)
    QrCand last = ~0ull;
    for (int r = 0; r < a.K; ++r) {
        QrCand mine = 0;
        for (int i = tid; i < n; i += NT) {
            const float l = (float)x[i];
            const QrCand c = l > -INFINITY ? qr_cand(qr_float_key(l + 0.0f), first + i) : 0ull;
            if (c < last && c > mine) mine = c;
        }
        for (int off = 32; off > 0; off >>= 1) {
            const QrCand o = __shfl_xor(mine, off);
            mine = o > mine ? o : mine;
        }
        if (lane == 0) wave_best[wave] = mine;
        __syncthreads();
        for (int w = 0; w < NW; ++w) mine = wave_best[w] > mine ? wave_best[w] : mine;
        __syncthreads();
        if (tid == 0) out[r] = mine;
        last = mine;   // 0: nothing is smaller, the ranks that follow stay empty
    }
}

// What turns a row's logits into values: logit - lse = (logit - top) - log(sum of exp(logit - top)).  With the two apart also
// logits of the type's lowest value, next to which the logarithm vanishes, give what they mean.
struct QrRowValue {
    double score, top, log_sum;   // log_sum NaN: no candidates
    __device__ __forceinline__ QrValue operator()(float logit) const { return value_word(score + (((double)logit - top) - log_sum)); }
};

// Long rows, second launch.  Grid: one workgroup of NT = 256 or 1024 threads an utterance.  HELD: what the lists have in all fits four
// to a thread, which are fetched at once and kept (otherwise they are read in every pass).
template <int NT, bool HELD>
__global__ __launch_bounds__(NT) void select_beam_kernel(const QrSelectArgs a)
{
    __shared__ QrPickList list;
    __shared__ QrRowValue rows[64];
    __shared__ unsigned group_best[256];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int64_t row0 = (int64_t)b * a.W;
    const int per = a.n_parts * a.K, total = a.W * per;
    // Groups for the bound: a thread, or four neighbours, with every 256th candidate, each time 73 further on: the best ranks of the
    // lists, which make up most of what is taken, are spread over the groups (n_out 64 of 64 hypotheses: 80 candidates pass the
    // bound; with four ranks that follow one another to a group 380 would)
    auto index = [&](int q) { const int block = NT == 256 ? q : q * 4 + (tid & 3); return ((NT == 256 ? tid : tid >> 2) - 73 * block & 255) + 256 * block; };
    QrCand held[4];
    if (HELD) {
#pragma unroll
        for (int q = 0; q < 4; ++q) held[q] = a.cands[row0 * per + (index(q) < total ? index(q) : 0)];
    }
    if (tid == 0) list.n = 0;
    // four threads to a row
    if (tid < 4 * a.W) {
        const int64_t row = row0 + (tid >> 2);
        double ls = NAN;
        float top = -INFINITY;
        if (reads_logits(a, row)) {
            ls = 0.0;
            if (a.log_softmax) {
                const QrPartHead *h = a.heads + row * a.n_parts;
                for (int i = tid & 3; i < a.n_parts; i += 4) top = fmaxf(top, h[i].top);
                top = fmaxf(top, __shfl_xor(top, 1));
                top = fmaxf(top, __shfl_xor(top, 2));
                for (int i = tid & 3; i < a.n_parts; i += 4) ls += h[i].top > -INFINITY ? h[i].sum * (double)qr_exp(h[i].top - top) : h[i].sum;
                ls += __shfl_xor(ls, 1);
                ls += __shfl_xor(ls, 2);
                ls = top > -INFINITY ? log(ls) : NAN;
            }
        }
        if ((tid & 3) == 0) rows[tid >> 2] = {(double)a.score[row], a.log_softmax ? (double)top : 0.0, ls};
    }
    __syncthreads();
    auto pick = [&](int i, QrCand c) -> QrPick {
        const int w = i / per;
        const QrRowValue row = rows[w];
        return {row.log_sum == row.log_sum && c ? row(qr_cand_value(c)) : 0ull, c, w};   // (rows that were not asked for hold anything)
    };
    QrPick kept[4];
    if (HELD) {
#pragma unroll
        for (int q = 0; q < 4; ++q) kept[q] = index(q) < total ? pick(index(q), held[q]) : QrPick{0ull, 0ull, 0};
    }
    auto each = [&](auto &&visit) {
        if (HELD) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (kept[q].v) visit(kept[q]);
        } else {
#pragma unroll 4
            for (int q = 0; q * NT < total; ++q) {
                const int i = index(q);
                const QrPick p = i < total ? pick(i, a.cands[row0 * per + i]) : QrPick{0ull, 0ull, 0};
                if (p.v) visit(p);
            }
        }
        if (a.finished && tid < a.W && a.finished[row0 + tid]) {
            const QrPick p = {value_word((double)a.score[row0 + tid]), qr_cand(1u, a.end_token), tid};
            if (p.v) visit(p);
        }
    };
    unsigned top = 0u;
    each([&](const QrPick &p) { top = (unsigned)(p.v >> 32) > top ? (unsigned)(p.v >> 32) : top; });
    if (NT == 256) {
        group_best[tid] = top;
    } else {
        const unsigned k = quad_max(top);
        if ((tid & 3) == 0) group_best[tid >> 2] = k;
    }
    __syncthreads();
    unsigned g[4], most = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = group_best[i * 64 + lane];
        most = g[i] > most ? g[i] : most;
    }
    const unsigned T = bound_of(g, qr_wave_reduce_u32<true>(most), a.K, a.K + a.K / 4);
    if (top >= T)
        each([&](const QrPick &p) {
            if ((unsigned)(p.v >> 32) >= T) push(list, p);
        });
    __syncthreads();
    write_ranks<NT>(a, b, list, each);
}

// Short rows: one launch, one workgroup of 16 waves an utterance, wave i takes the rows i, i + 16, ...; a row has at most 64 * NV * V
// logits.  Bound by its chain of steps, of 0.3 to 1 us each: 5.3 us for 1 x 4 x 1000 fp32, 9.8 for 64 x 16 x 1000 bf16.
template <class T, int NV>
__global__ __launch_bounds__(1024) void select_short_kernel(const QrSelectArgs a)
{
    constexpr int V = QrVec<T>::N;
    __shared__ QrPickList list;
    __shared__ QrRowValue rows[64];
    __shared__ unsigned group_best[256];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = (int64_t)b * a.W;
    const T *x = (const T *)a.logits + row0 * a.ld;
    if (tid == 0) list.n = 0;
    QrLogits<T, NV> f;
    unsigned best = 0u;
    for (int w = wave; w < a.W; w += 16) {   // uniform in a wave
        QrRowValue row = {(double)a.score[row0 + w], 0.0, NAN};
        if (reads_logits(a, row0 + w)) {
            f.load(x + w * a.ld, a.V, lane, 64);
            const float largest = f.largest();
            row.log_sum = 0.0;
            if (a.log_softmax) {
                const unsigned k = qr_wave_reduce_u32<true>(logit_key(largest));
                const float top = k ? qr_key_float(k) : -INFINITY;
                row.top = (double)top;
                row.log_sum = log(wave_sum((double)f.sum_exp(top)));   // (of -inf alone: NaN)
            }
            if (largest > -INFINITY) {
                const unsigned k = (unsigned)(row(largest) >> 32);
                best = k > best ? k : best;
            }
        } else if (is_finished(a, row0 + w) && lane == 0) {
            const unsigned k = (unsigned)(value_word(row.score) >> 32);
            best = k > best ? k : best;
        }
        if (lane == 0) rows[w] = row;
    }
    if (a.W <= 4) {   // groups: lanes of 4 waves, or quads of 16
        if (wave < 4) group_best[tid] = best;
    } else {
        best = quad_max(best);
        if ((lane & 3) == 0) group_best[tid >> 2] = best;
    }
    __syncthreads();
    unsigned g[4], most = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = group_best[i * 64 + lane];
        most = g[i] > most ? g[i] : most;
    }
    const unsigned Tk = bound_of(g, qr_wave_reduce_u32<true>(most), a.K, a.K + a.K / 4);
    for (int w = wave; w < a.W; w += 16) {
        const QrRowValue row = rows[w];
        if (row.log_sum == row.log_sum) {
            if (a.W > 16) f.load(x + w * a.ld, a.V, lane, 64);
            // the bound as a logit of this row, and a little lower, by 1e-6 of it (its rounding to fp32) and by what the sums to the value and
            // back are rounded by, a few halves of 2^-52 of the largest number in them (where they cancel that is all there is: 1 - 1e-20 is 1);
            // where it has none every logit passes.  What passes is held against the bound itself.
            const double bound = word_value((QrValue)Tk << 32);
            const double at = Tk ? ((bound - row.score) + row.log_sum) + row.top : -INFINITY;
            const double less = 1e-6 * fabs(at) + 0x1p-48 * (fabs(bound) + fabs(row.score) + fabs(row.log_sum) + fabs(row.top));
            const float least = at == at ? fmaxf((float)(at - less), -FLT_MAX) : -FLT_MAX;
            f.hits(least, [&](float l, int i) {
                const QrPick p = {row(l), qr_cand(qr_float_key(l + 0.0f), ((i / V) * 64 + lane) * V + i % V), w};
                if ((unsigned)(p.v >> 32) >= Tk && p.v) push(list, p);
            });
        } else if (lane == 0 && is_finished(a, row0 + w)) {
            const QrPick p = {value_word(row.score), qr_cand(1u, a.end_token), w};
            if ((unsigned)(p.v >> 32) >= Tk && p.v) push(list, p);
        }
    }
    __syncthreads();
    write_ranks<1024>(a, b, list, [&](auto &&visit) {
        for (int w = wave; w < a.W; w += 16) {
            const QrRowValue row = rows[w];
            if (row.log_sum == row.log_sum) {
                for (int c = lane; c < a.V; c += 64) {
                    const float l = (float)x[w * a.ld + c];
                    const QrPick p = {row(l), qr_cand(qr_float_key(l + 0.0f), c), w};
                    if (p.v) visit(p);
                }
            } else if (lane == 0 && is_finished(a, row0 + w)) {
                const QrPick p = {value_word(row.score), qr_cand(1u, a.end_token), w};
                if (p.v) visit(p);
            }
        }
    });
}

// How rows are cut.  One launch for rows of up to 512 logits (16 x 32 x 300 fp32 10.0 us, two launches 13.3) and of up to 2048 unless
// wide beams leave most of the device idle (16 x 16 x 2000 9.4 us, two launches 11.0; 64 x 64 x 2000 25.5 and 34; but 1 x 64 x 2000 21.9
// and 15.6, 16 x 32 x 600 16.7 and 13.4).  Whole rows of up to 8192 to 256 threads, longer ones in stretches of up to 16384 to 512
// (64 x 16 x 32000 bf16, n_out 16: 24.8 us, by 8192 25.7; 16 x 16 x 32000 fp32, n_out 32: 17.6 and 19.6; 4 x 8 x 131072 12.1
// and 13.1; only 2 x 2 x 50000 is better by 8192: 9.4 and 9.1).
constexpr int SHORT = 2048, STRETCH = 16384, FEW_ROWS = 1024;
bool always_one_launch(int W, int V) { return V <= 512 || (V <= SHORT && W <= 24); }   // for any number of rows
bool one_launch(int64_t rows, int W, int V) { return always_one_launch(W, V) || (V <= SHORT && rows > FEW_ROWS); }
void plan_select(int V, int &n_parts, int &part)
{
    n_parts = (V + STRETCH - 1) / STRETCH;
    part = qr_round_up((V + n_parts - 1) / n_parts, 8);
    n_parts = (V + part - 1) / part;
}

bool select_sizes_ok(int32_t B, int32_t W, int32_t V, int32_t K)
{
    return B >= 0 && W > 0 && V > 0 && K > 0 && W <= 64 && K <= MAX_OUT && (int64_t)W * V <= INT32_MAX && V <= 1 << 30 && B <= 1 << 21;   // (a grid has less than 2^32 threads)
}

size_t heads_bytes(int64_t rows, int n_parts) { return ((size_t)rows * n_parts * sizeof(QrPartHead) + 255) / 256 * 256; }

template <class T>
void launch_select(QrSelectArgs &a, void *workspace, hipStream_t st)
{
    constexpr int V = QrVec<T>::N;
    const int64_t rows = (int64_t)a.B * a.W;
    if (one_launch(rows, a.W, a.V)) {
        if (a.V <= 512) select_short_kernel<T, 512 / 64 / V><<<a.B, 1024, 0, st>>>(a);
        else select_short_kernel<T, SHORT / 64 / V><<<a.B, 1024, 0, st>>>(a);
        return;
    }
    plan_select(a.V, a.n_parts, a.part);
    a.heads = (QrPartHead *)workspace;
    a.cands = (QrCand *)((char *)workspace + heads_bytes(rows, a.n_parts));
    const dim3 grid(a.n_parts, (unsigned)(rows < 32768 ? rows : 32768), (unsigned)((rows + 32767) / 32768));
    if (a.V <= 8192) select_parts_kernel<T, 8192 / 256 / V, 256><<<grid, 256, 0, st>>>(a);
    else select_parts_kernel<T, 16384 / 512 / V, 512><<<grid, 512, 0, st>>>(a);
    const int64_t total = (int64_t)a.W * a.n_parts * a.K;
    if (total <= 1024) select_beam_kernel<256, true><<<a.B, 256, 0, st>>>(a);
    else if (total <= 4096) select_beam_kernel<1024, true><<<a.B, 1024, 0, st>>>(a);
    else select_beam_kernel<1024, false><<<a.B, 1024, 0, st>>>(a);
}

}  // namespace

extern "C" size_t qrnnt_beam_select_workspace(int32_t B, int32_t W, int32_t V, int32_t n_out)
{
    if (!select_sizes_ok(B, W, V, n_out)) return 0;
    // what the largest call within these sizes takes: a smaller batch may go in two launches where this one goes in one
    int64_t rows = (int64_t)(B > 0 ? B : 1) * W;
    if (always_one_launch(W, V)) return 256;   // (not used)
    if (V <= SHORT && rows > FEW_ROWS) rows = FEW_ROWS;
    const int n_parts = (V + STRETCH - 1) / STRETCH;
    return heads_bytes(rows, n_parts) + (size_t)rows * n_parts * n_out * sizeof(QrCand);
}

extern "C" qrnnt_status qrnnt_beam_select(const float *score, const void *logits, int32_t dtype, int64_t ld, int32_t log_softmax,
                                          const uint8_t *finished, int32_t end_token, int32_t B, int32_t W, int32_t V,
                                          int32_t n_out, int32_t *parent_out, int32_t *token_out, float *score_out,
                                          uint8_t *finished_out, void *workspace, size_t workspace_bytes, void *stream)
{
    QR_REQUIRE(qr_is_dtype(dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(B >= 0 && W > 0 && V > 0 && n_out > 0 && ld >= V, QRNNT_ERR_SHAPE);
    QR_REQUIRE(select_sizes_ok(B, W, V, n_out) && qr_pitch_ok((int64_t)B * W, ld), QRNNT_ERR_UNSUPPORTED);
    QR_REQUIRE(finished == nullptr || (end_token >= 0 && end_token < V), QRNNT_ERR_RANGE);
    if (B == 0) return QRNNT_OK;
    QR_REQUIRE(score && logits && parent_out && token_out && score_out && workspace, QRNNT_ERR_NULL);
    QR_REQUIRE(qr_aligned(score, 4) && qr_aligned(logits, qr_dtype_size(dtype)) && qr_aligned(parent_out, 4) && qr_aligned(token_out, 4) &&
                   qr_aligned(score_out, 4) && qr_aligned(workspace, 256), QRNNT_ERR_ALIGN);
    QR_REQUIRE(workspace_bytes >= qrnnt_beam_select_workspace(B, W, V, n_out), QRNNT_ERR_WORKSPACE);
    QrSelectArgs a = {};
    a.score = score;  a.logits = logits;  a.ld = ld;  a.finished = finished;  a.log_softmax = log_softmax;  a.end_token = end_token;
    a.B = B;  a.W = W;  a.V = V;  a.K = n_out;
    a.parent_out = parent_out;  a.token_out = token_out;  a.score_out = score_out;  a.finished_out = finished_out;
    if (dtype == QRNNT_F32) launch_select<float>(a, workspace, (hipStream_t)stream);
    else if (dtype == QRNNT_F16) launch_select<_Float16>(a, workspace, (hipStream_t)stream);
    else launch_select<__bf16>(a, workspace, (hipStream_t)stream);
    return qr_launch_status();
}
