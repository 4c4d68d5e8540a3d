// Scores of given tokens, from logits: log probability of a row's token, entropy of the row, its best alternatives, in one pass
// over the logits.
//
// With S = sum 2^(x L - r), U = sum 2^(x L - r)(x L - r), L = log2(e), for any r:  log P(x) = (x L - r) / L - log S,
// entropy = log S - U / (L S).  A wave takes the largest logit of the first that it reads for r, a product, a sum, an exponential and
// two more sums a logit then do; where a logit passes r by far (a sum of 2^12) sums move to a larger one.  Lanes add up at the end of
// the row, in fp32.  What fp32 cannot hold this way (a largest logit beyond 1.1e7 in magnitude, where x L is no longer
// known to 1, infinities, NaN, nothing but -inf) shows in S and U and is read again, with x - max formed first.
//
// The best alternatives: the n-th largest of groups of the logits that are read first bounds the n-th best from below.  What reaches the
// bound goes to a list in LDS, of which the n best are kept where it fills, and their smallest becomes the bound; at the end a
// candidate's rank is how many are better.
#include <float.h>
#include <type_traits>

#include "elem.h"
#include "kernels.h"
#include "select.h"

namespace {

constexpr int MAX_TOP = 64, CAP = 256;        // ranks; candidates in a wave's list
constexpr int LIST = 1024, VECS = 512;       // candidates and vectors in a workgroup's lists
constexpr int MAX_PARTS = 16, FEW_RANKS = 24;
constexpr float LOG2E = 1.4426950408889634f, FAR = -300.0f;   // 2^FAR is 0 in fp32
constexpr float MOST = 0x1p24f;                               // r stays within, so that it is less than 1 from the x L that it was rounded from
constexpr double LN2 = 0.69314718055994530942;
constexpr double UNIT = 1.0 / (double)LOG2E;                  // of x L - r, with the L that the sums take (2^-26 from log2(e), of which 1e9 would show)

// ln s of a positive number to 2^-32: s = 2^e m with m in [2/3, 4/3), ln m = 2 (z + z^3 / 3 + z^5 / 5 + ...) with z = (m - 1) / (m + 1), at most
// 1/5 in magnitude; behind z^11 / 11 less than 2^-32 is left out.  (log(), exact to the last bit, takes
// four times the instructions, a quarter of a short row's: 16384 x 64 fp32 without alternatives 8.1 us with it, 6.6 without.)
__device__ __forceinline__ double log_of_sum(double s)
{
    double m = __builtin_amdgcn_frexp_mant(s);   // [1/2, 1)
    int e = __builtin_amdgcn_frexp_exp(s);
    const bool low = m < 2.0 / 3.0;
    m = low ? 2.0 * m : m;
    e = low ? e - 1 : e;
    const double b = m + 1.0, r0 = (double)__builtin_amdgcn_rcpf((float)b), r = fma(fma(-b, r0, 1.0), r0, r0);   // (off by 2^-44)
    const double z = (m - 1.0) * r, q = z * z;
    const double p = fma(fma(fma(fma(fma(q, 1.0 / 11, 1.0 / 9), q, 1.0 / 7), q, 1.0 / 5), q, 1.0 / 3), q, 1.0);
    return fma((double)e, LN2, 2.0 * z * p);
}

// A part's sums.
struct QrScoresSum {
    double r, s, u;
    // to an r that is not below
    __device__ __forceinline__ void move(double to)
    {
        const double d = fmax(r - to, (double)FAR), c = (double)__builtin_amdgcn_exp2f((float)d);
        u = c * (u + d * s);
        s *= c;
        r = to;
    }
    // (both: where d is some 120, e d passes fp32 before e does)
    __device__ __forceinline__ bool finite() const { return s < INFINITY && fabs(u) < INFINITY; }
    // Whether a logit lies at r: always, but where all are -inf or beyond MOST.
    __device__ __forceinline__ bool some() const { return s >= 0.5; }
};

struct QrScoresArgs {
    const void *logits;
    int64_t ld;
    const int32_t *token;
    int rows, V, n;
    int n_parts, part;       // parts of a row, and their length
    float *logp, *entropy;
    int32_t *top_token;
    float *top_logp;
    QrScoresSum *heads;      // [rows][n_parts]
    QrCand *cands;           // [rows][n_parts][n], 0: none
};

// A row's token and its logit, fetched before the row is read.
struct QrScoresToken {
    int t = -1;
    float x = 0.0f;
    template <class T>
    __device__ __forceinline__ void load(const QrScoresArgs &a, int64_t row)
    {
        if (!a.logp) return;
        t = a.token[row];
        x = (float)((const T *)a.logits)[row * a.ld + (t >= 0 && t < a.V ? t : 0)];
    }
};

// Values of a row's logits from its sums.
struct QrScoresRow {
    double r, log_s, entropy;
    bool none, bad;   // no token can be; a logit is NaN or +inf
    QrScoresRow() = default;
    __device__ __forceinline__ explicit QrScoresRow(const QrScoresSum &a)
    {
        r = a.r;
        none = a.s == 0.0;
        bad = !(a.s == a.s);
        log_s = log_of_sum(a.s);
        entropy = none ? 0.0 : log_s - UNIT * (a.u / a.s);
    }
    __device__ __forceinline__ float logp(float logit) const { return none ? -INFINITY : (float)(UNIT * ((double)logit * (double)LOG2E - r) - log_s); }
    __device__ __forceinline__ void write(const QrScoresArgs &a, int64_t row, const QrScoresToken &t) const
    {
        if (a.logp) a.logp[row] = t.t < 0 ? 0.0f : t.t >= a.V ? NAN : logp(t.x);
        if (a.entropy) a.entropy[row] = (float)entropy;
    }
    __device__ __forceinline__ void write_rank(const QrScoresArgs &a, int64_t row, int rank, QrCand c) const
    {
        const bool some = c != 0ull && !bad;
        a.top_token[row * a.n + rank] = some ? qr_cand_index(c) : -1;
        a.top_logp[row * a.n + rank] = some ? logp(qr_cand_value(c)) : -INFINITY;
    }
};

// Four vectors of a lane out of 256 that follow one another; -inf behind the end.
template <class T>
struct QrChunk {
    static constexpr int V = QrVec<T>::N, LEN = 256 * V, PER = 4 * V;
    v4i raw[4];
    // Whether any lane's vector v holds one of n logits (v = 0: as if it did).
    static __device__ __forceinline__ bool holds(int v, int n) { return v == 0 || v * 64 * V < n; }
    __device__ __forceinline__ void load(const T *x, int n, int lane)
    {
        if (n >= LEN) {   // uniform
#pragma unroll
            for (int v = 0; v < 4; ++v) raw[v] = __builtin_bit_cast(v4i, *(const typename QrVec<T>::any *)(x + (v * 64 + lane) * V));
            return;
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int c = (v * 64 + lane) * V;
            typename QrVec<T>::type u;
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] = (T)-INFINITY;
            raw[v] = __builtin_bit_cast(v4i, u);
            if (!holds(v, n)) continue;   // uniform
            if (c + V <= n) {
                raw[v] = __builtin_bit_cast(v4i, *(const typename QrVec<T>::any *)(x + c));
            } else if (c < n) {
#pragma unroll
                for (int i = 0; i < V; ++i) u[i] = c + i < n ? x[c + i] : (T)-INFINITY;
                raw[v] = __builtin_bit_cast(v4i, u);
            }
        }
    }
    __device__ __forceinline__ float at(int i) const
    {
        const unsigned w = (unsigned)raw[i / V][i % V * (int)sizeof(T) / 4];
        if constexpr (sizeof(T) == 4) return __uint_as_float(w);
        if constexpr (std::is_same<T, __bf16>::value) return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w >> 16 : w));
    }
    // What follows widens the logits again: kept in fp32 from one use to the next they would take other waves' registers.
    __device__ __forceinline__ void fresh()
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) asm volatile("" : "+v"(raw[v]));
    }
};

typedef __attribute__((address_space(3))) QrCand *QrLdsList;   // (for functions that are not inlined)

__device__ __forceinline__ int lanes_below(unsigned long long m)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
}
// (keys up to there are those of -inf and below)
__device__ __forceinline__ float least_of(unsigned key) { return key > 0x00800000u ? qr_key_float(key) : -FLT_MAX; }
__device__ __forceinline__ float wave_max(float v) { return qr_key_float(qr_wave_reduce_u32<true>(qr_float_key(v))); }   // (v is not NaN)
__device__ __forceinline__ float wave_add(float v)   // in all lanes: within rows of 16, then over the rows
{
#define QR_DPP_ADD(ctrl, rmask) v += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), ctrl, rmask, 0xf, false))
    QR_DPP_ADD(0x111, 0xf);   // row_shr:1
    QR_DPP_ADD(0x112, 0xf);   // row_shr:2
    QR_DPP_ADD(0x114, 0xf);   // row_shr:4
    QR_DPP_ADD(0x118, 0xf);   // row_shr:8
    QR_DPP_ADD(0x142, 0xa);   // row_bcast:15 into rows 1 and 3
    QR_DPP_ADD(0x143, 0xc);   // row_bcast:31 into rows 2 and 3
#undef QR_DPP_ADD
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}
__device__ __forceinline__ float limited(float r) { return fminf(fmaxf(r, -MOST), MOST); }

// A wave keeps the n best of a list in LDS, or up to `enough` while that needs no look at indices; returns the key that n of them reach
// (0: there are fewer).  (The bound is the n-th largest key itself unless no more than `enough` reach it: what is left is never more than that.)
template <int ROOM, class List>
__device__ __forceinline__ unsigned keep_best(List list, int &count, int n, int enough, int lane)
{
    QrCand e[ROOM / 64];
    unsigned g[ROOM / 64], top = 0u;
#pragma unroll
    for (int j = 0; j < ROOM / 64; ++j) {
        e[j] = lane + 64 * j < count ? list[lane + 64 * j] : 0ull;
        g[j] = (unsigned)(e[j] >> 32);
        top = g[j] > top ? g[j] : top;
    }
    const unsigned T = qr_bound_of(g, qr_wave_reduce_u32<true>(top), n, enough);
    if (T == 0u) return 0u;
    int above = 0, equal = 0;
#pragma unroll
    for (int j = 0; j < ROOM / 64; ++j) {
        above += (int)__popcll(__ballot(g[j] > T));
        equal += (int)__popcll(__ballot(g[j] == T));
    }
    unsigned low = 0u;   // of the equal ones: the words (complements of the indices) from here on
    if (above + equal > enough) {
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned trial = low | (1u << bit);
            int some = 0;
#pragma unroll
            for (int j = 0; j < ROOM / 64; ++j) some += (int)__popcll(__ballot(g[j] == T && (unsigned)e[j] >= trial));
            if (above + some >= n) low = trial;
        }
    }
    int at = 0;
#pragma unroll
    for (int j = 0; j < ROOM / 64; ++j) {
        const bool stays = g[j] > T || (g[j] == T && (unsigned)e[j] >= low);
        const unsigned long long m = __ballot(stays);
        if (stays) list[at + lanes_below(m)] = e[j];
        at += (int)__popcll(m);
    }
    count = at;
    __builtin_amdgcn_wave_barrier();
    return T;
}

// A wave's sums and best logits, as it goes through a row.  All but the lanes' sums is uniform.
template <class T>
struct QrScoresWave {
    static constexpr int V = QrVec<T>::N, PER = QrChunk<T>::PER;
    QrChunk<T> now;
    float best[4], largest;   // of each vector, of all four (not NaN)
    float r = -MOST;
    double s = 0.0, u = 0.0;

    // n: logits from the chunk's start on; VECS: of its vectors
    template <int VECS = 4>
    __device__ __forceinline__ void find_best(int n)
    {
        now.fresh();
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            best[v] = -INFINITY;
            if (v >= VECS || !QrChunk<T>::holds(v, n)) continue;   // uniform
            best[v] = now.at(v * V);
#pragma unroll
            for (int i = 1; i < V; ++i) best[v] = fmaxf(best[v], now.at(v * V + i));
        }
        largest = fmaxf(-INFINITY, fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3])));
    }
    // from the first vectors, so that r is the same whether the others' largest are known or not
    __device__ __forceinline__ void start() { r = limited(LOG2E * wave_max(fmaxf(-INFINITY, best[0]))); }
    __device__ __forceinline__ void add_chunk(int n, float &cs, float &cu)
    {
        cs = cu = 0.0f;
        now.fresh();
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (!QrChunk<T>::holds(v, n)) continue;   // uniform
#pragma unroll
            for (int i = v * V; i < (v + 1) * V; ++i) {
                const float d = fmaf(now.at(i), LOG2E, -r), e = __builtin_amdgcn_exp2f(d);
                cs += e;
                cu = fmaf(e, fmaxf(d, FAR), cu);
            }
        }
    }
    template <bool FOUND>
    __device__ __forceinline__ void add(int n)
    {
        float cs, cu;
        add_chunk(n, cs, cu);
        if (__ballot(!(cs < 0x1p12f))) {
            if (!FOUND) find_best(n);
            const float to = limited(LOG2E * wave_max(largest));
            if (to > r) {
                QrScoresSum moved = {(double)r, s, u};
                moved.move((double)to);
                r = to;
                s = moved.s;
                u = moved.u;
                add_chunk(n, cs, cu);
            }
        }
        s += (double)cs;
        u += (double)cu;
    }
    __device__ __forceinline__ QrScoresSum sum() const { return {(double)r, (double)wave_add((float)s), (double)wave_add((float)u)}; }
    // Which of a lane's logits are not below `least`, as bits.
    __device__ __forceinline__ unsigned from(float least)
    {
        unsigned mask = 0u;
        now.fresh();
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (!__ballot(best[v] >= least)) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) mask |= now.at(v * V + i) >= least ? 1u << (v * V + i) : 0u;
        }
        return mask;
    }
    // The logit of the lowest bit of `mask` and its place in the chunk at x; all: the bits before any was taken.  The only one of a
    // vector is the vector's largest; where there are more (seldom) they are read again, which takes less code than a way for each register.
    __device__ __forceinline__ float pop(unsigned &mask, unsigned all, const T *x, int lane, int &place) const
    {
        const int b = __builtin_ctz(mask), v = b / V;
        mask &= mask - 1u;
        place = (v * 64 + lane) * V + b % V;
        const float b0 = best[0], b1 = best[1], b2 = best[2], b3 = best[3];   // (values: a choice of places would put them into memory)
        float f = v == 0 ? b0 : v == 1 ? b1 : v == 2 ? b2 : b3;
        if (__popc(all & (((1u << V) - 1u) << (v * V))) > 1) f = (float)x[place];
        return f;
    }
    // take(logit, place in the chunk at x) for the logits from `least` on.
    template <class Take>
    __device__ __forceinline__ void hits(float least, const T *x, int lane, Take &&take)
    {
        if (!__ballot(largest >= least)) return;
        const unsigned all = from(least);
        for (unsigned mask = all; mask != 0u;) {
            int i;
            const float f = pop(mask, all, x, lane, i);
            take(f, i);
        }
    }
    // Vectors that hold a logit from `least` on into a workgroup's list, while it has room.  at: index of the chunk's first logit.
    __device__ __forceinline__ void vectors_to(v4i *vecs, int *index, int *n_vecs, int room, float least, int at, int lane) const
    {
        if (!__ballot(largest >= least)) return;
        unsigned long long m[4];
        int some = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            m[v] = __ballot(best[v] >= least);
            some += (int)__popcll(m[v]);
        }
        int to = 0;
        if (lane == 0) to = atomicAdd(n_vecs, some);
        to = __builtin_amdgcn_readfirstlane(to);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int mine = to + lanes_below(m[v]);
            if (best[v] >= least && mine < room) {
                vecs[mine] = now.raw[v];
                index[mine] = at + (v * 64 + lane) * V;
            }
            to += (int)__popcll(m[v]);
        }
    }
    // Logits from the key on into a wave's list, which never overflows: where it is full its n best are kept.  first: index of the chunk's first logit.
    template <class List>
    __device__ __forceinline__ void hits_to(List list, int &count, unsigned &key, int n, const T *x, int first, int lane)
    {
        float least = least_of(key);
        if (!__ballot(largest >= least)) return;
        const unsigned all = from(least);
        for (unsigned mask = all; __ballot(mask != 0u);) {   // uniform
            int i = 0;
            float f = -INFINITY;
            if (mask != 0u) f = pop(mask, all, x, lane, i);
            unsigned long long m = __ballot(f >= least);
            if (count + (int)__popcll(m) > CAP) {
                // (n of the list reach the key, but what is left of these logits may lie in front of them)
                const unsigned k = keep_best<CAP>(list, count, n, n + n / 4, lane);
                key = k > key ? k : key;
                least = least_of(key);
                m = __ballot(f >= least);
            }
            if (f >= least) list[count + lanes_below(m)] = qr_cand(qr_float_key(f + 0.0f), first + i);
            count += (int)__popcll(m);
        }
        __builtin_amdgcn_wave_barrier();
        if (count >= 3 * n + 48) {
            // what this wave has not read yet lies behind: to be among the best it has to be larger
            const unsigned k = keep_best<CAP>(list, count, n, n + n / 4, lane) + 1u;
            key = k > key ? k : key;
        }
    }
};

// The bound that groups of a wave's logits give.  Few ranks: a lane's are a group, and up to twice as many may reach the bound, which makes
// the search shorter; of many ranks counting them would take longer (1024 x 32000 bf16, 64 ranks 35 us, with a quarter more at most 28).
template <class T>
__device__ __forceinline__ unsigned first_bound(const QrScoresWave<T> &w, int n)
{
    if (n <= FEW_RANKS) {
        const unsigned g[1] = {qr_logit_key(w.largest)};
        return qr_bound_of(g, qr_wave_reduce_u32<true>(g[0]), n, 2 * n);
    }
    unsigned g[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) g[v] = qr_logit_key(w.best[v]);
    return qr_bound_of(g, qr_wave_reduce_u32<true>(qr_logit_key(w.largest)), n, n + n / 4);
}

// Sums of a row's part that are good for any logits: relative to its largest one.  WPR waves of a workgroup, `most` in LDS.
// (A part that holds nothing but masks of -1e9 comes here: 64 x 131072 fp32, the last of four parts masked so, 16.8 us, with masks of -1e4
// 7.5.  Differences formed first in the pass itself, for logits beyond MOST, leave no registers to the others: 1024 x 32000 bf16 with 16
// alternatives 22.5 us instead of 20.0; this function by whole vectors 16384 x 32000 without any 224 instead of 169.)
template <class T, int WPR>
__device__ __attribute__((noinline)) QrScoresSum sums_of_any(const T *x, int n, int wave, int lane, float *most)
{
    float m = -INFINITY;
    bool nan = false;
    for (int c = wave * 64 + lane; c < n; c += WPR * 64) {
        const float f = (float)x[c];
        m = fmaxf(m, f);
        nan = nan || !(f < INFINITY);
    }
    m = wave_max(m);
    nan = __ballot(nan) != 0ull;
    if (WPR > 1) {
        if (lane == 0) most[wave] = nan ? INFINITY : m;
        __syncthreads();
        for (int w = 0; w < WPR; ++w) m = fmaxf(m, most[w]);
        nan = !(m < INFINITY);
    }
    if (nan) return {0.0, NAN, NAN};
    if (m == -INFINITY) return {0.0, 0.0, 0.0};
    QrScoresSum sum = {(double)m * (double)LOG2E, 0.0, 0.0};
    for (int c = wave * 64 + lane; c < n; c += WPR * 64) {
        const float d = LOG2E * ((float)x[c] - m), e = __builtin_amdgcn_exp2f(d);
        sum.s += (double)e;
        sum.u += (double)(e * fmaxf(d, FAR));
    }
    return {sum.r, qr_wave_sum(sum.s), qr_wave_sum(sum.u)};
}

// A wave to a row: many rows, or short ones.  Grid: y (and z) = four rows.
// Bound by what its instructions take, and by memory (16384 x 32000 bf16, 1.05 GB, 16 alternatives: 225 us, 4.7 TB/s).  Without
// alternatives four waves to a SIMD (the same rows 190 us, with eight and their fewer registers 198).
template <class T, bool TOP>
__global__ __launch_bounds__(256, TOP ? 8 : 4) void scores_wave_kernel(const QrScoresArgs a)
{
    constexpr int LEN = QrChunk<T>::LEN;
    __shared__ QrCand lists[TOP ? 4 : 1][TOP ? CAP : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = (blockIdx.y + (int64_t)blockIdx.z * 32768) * 4 + wave;
    if (row >= a.rows) return;
    const int n = a.V;
    const T *x = (const T *)a.logits + row * a.ld;
    QrScoresWave<T> w;
    w.now.load(x, n, lane);
    QrScoresToken token;
    token.load<T>(a, row);
    QrCand *list = lists[TOP ? wave : 0];
    int count = 0;
    unsigned key = 0u;
    for (int at = 0;; at += LEN) {
        const bool more = n - at > LEN;
        QrChunk<T> next;
        if (more) next.load(x + at + LEN, n - at - LEN, lane);
        if (TOP) w.find_best(n - at);
        else if (at == 0) w.template find_best<1>(n);   // (enough to begin with)
        if (at == 0) w.start();
        w.template add<TOP>(n - at);
        if (TOP) {
            if (at == 0) key = first_bound(w, a.n);
            w.hits_to(list, count, key, a.n, x + at, at, lane);
        }
        if (!more) break;
        w.now = next;
    }
    QrScoresSum sum = w.sum();
    if (!sum.some() || !sum.finite()) sum = sums_of_any<T, 1>(x, n, 0, lane, nullptr);
    const QrScoresRow values(sum);
    if (lane == 0) values.write(a, row, token);
    if (TOP) {
        if (count > 128) keep_best<CAP>(list, count, a.n, a.n, lane);
        const QrCand c0 = lane < count ? list[lane] : 0ull, c1 = lane + 64 < count ? list[lane + 64] : 0ull;
        int r0 = 0, r1 = 0;
        if (count <= 64) {   // uniform
#pragma unroll 4
            for (int j = 0; j < count; ++j) r0 += list[j] > c0 ? 1 : 0;
        } else {
#pragma unroll 4
            for (int j = 0; j < count; ++j) {
                const QrCand o = list[j];
                r0 += o > c0 ? 1 : 0;
                r1 += o > c1 ? 1 : 0;
            }
            if (c1 != 0ull && r1 < a.n) values.write_rank(a, row, r1, c1);
        }
        if (c0 != 0ull && r0 < a.n) values.write_rank(a, row, r0, c0);
        if (lane >= count && lane < a.n) values.write_rank(a, row, lane, 0ull);
    }
}

// What a list of the workgroup does not hold, because very many logits are equal or they rise: every wave finds the n best of what it
// reads by itself; one to a lane.
template <class T, int NW>
__device__ __attribute__((noinline)) QrCand best_of_any(const T *x, int len, int first, int n, int wave, int lane, QrLdsList list)
{
    QrScoresWave<T> w;
    int count = 0;
    unsigned key = 0u;
    for (int at = wave * QrChunk<T>::LEN; at < len; at += NW * QrChunk<T>::LEN) {
        w.now.load(x + at, len - at, lane);
        w.find_best(len - at);
        w.hits_to(list, count, key, n, x + at, first + at, lane);
    }
    if (count > n) keep_best<CAP>(list, count, n, n, lane);
    return lane < count ? list[lane] : 0ull;
}

// A workgroup of NW waves to a row or a part of one.  Grid: x = part of a row, y (and z) = row.
// Bound by a chain, not by memory: load, largest logit, bound, sums, list, ranks, one workgroup behind the other at each place on the
// device (1024 x 32000 bf16, 65.5 MB, 16 alternatives 20 us, of which vector units are busy 12; without alternatives 13.6, 4.8 TB/s).
// What the waves do on the chain is shared out: one searches the bound while the others add up, one joins the sums while the others
// rank.  Many long rows without alternatives are bound by memory (16384 x 32000 bf16, 1.05 GB, 168 us, 6.2 TB/s).
template <class T, int NW, bool TOP>
__global__ __launch_bounds__(64 * NW, 8) void scores_group_kernel(const QrScoresArgs a)
{
    constexpr int LEN = QrChunk<T>::LEN, BLOCK = NW * LEN, V = QrVec<T>::N;
    // Of 16-bit logits whole vectors go to a list first, which the workgroup looks through at the end: to look for a logit in a vector of
    // eight takes a wave 28 instructions, as many as to add it up (16 alternatives, 1024 x 32000 21.4 us so, 20.2 with vectors; 4096 x 32000
    // 62 and 58; of fp32, vectors of four, 4096 x 8000 25 and 29, 64 x 131072 13.0 and 13.5).
    constexpr bool VECTORS = sizeof(T) == 2;
    constexpr int ROOM = VECTORS ? VECS : LIST, EACH = (ROOM + 64 * NW - 1) / (64 * NW);   // of the first list; of it to a thread
    constexpr int POOL = !VECTORS || NW * CAP * 8 > VECS * 20 ? NW * CAP * 8 : VECS * 20;
    __shared__ __attribute__((aligned(16))) char pool[TOP ? POOL : 16];   // vectors and where they begin; or the lists of waves by themselves
    __shared__ QrCand list[TOP ? LIST : 1], ranked[TOP ? MAX_TOP : 1];
    v4i *vecs = (v4i *)pool;
    int *index = (int *)(pool + VECS * 16);
    __shared__ unsigned group_best[256], shared_key;
    __shared__ QrScoresSum sums[NW];
    __shared__ float most_of[NW];
    __shared__ int n_list, n_vecs;
    int &n_first = VECTORS ? n_vecs : n_list;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= a.rows) return;   // uniform
    const int first = blockIdx.x * a.part, n = a.V - first < a.part ? a.V - first : a.part;
    const T *x = (const T *)a.logits + row * a.ld + first;
    QrScoresWave<T> w;
    w.now.load(x + wave * LEN, n - wave * LEN, lane);   // (nothing behind the end is read)
    QrScoresToken token;
    if (a.n_parts == 1 && wave == 0) token.load<T>(a, row);
    if (TOP) {
        if (tid == 0) n_list = n_vecs = 0;
        if (tid < MAX_TOP) ranked[tid] = 0ull;
    }
    // every thread has a key: a bound from below of the n-th best, by the best keys of groups of threads.  The work is wave 0's, the
    // barrier behind it the caller's.
    auto find_bound = [&](unsigned k) {
        if (NW == 4) {
            group_best[tid] = k;
        } else if (NW == 8) {
            const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)k, 0xB1, 0xf, 0xf, true);   // the neighbour's
            if ((lane & 1) == 0) group_best[tid >> 1] = o > k ? o : k;
        } else {
            const unsigned four = qr_quad_max(k);
            if ((lane & 3) == 0) group_best[tid >> 2] = four;
        }
        __syncthreads();
        if (wave == 0) {
            unsigned g[4], one[1] = {0u};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                g[i] = group_best[i * 64 + lane];
                one[0] = g[i] > one[0] ? g[i] : one[0];
            }
            const unsigned top = qr_wave_reduce_u32<true>(one[0]);
            const unsigned bound = a.n <= FEW_RANKS ? qr_bound_of(one, top, a.n, 2 * a.n) : qr_bound_of(g, top, a.n, a.n + a.n / 4);
            if (lane == 0) shared_key = bound;
        }
    };
    auto push = [&](QrCand c) {
        const int to = atomicAdd(&n_list, 1);
        if (to < LIST) list[to] = c;
    };
    bool over = false;   // the list
    for (int at = 0;; at += BLOCK) {
        const bool more = n - at > BLOCK;
        const int mine = at + wave * LEN;
        QrChunk<T> next;
        if (more) next.load(x + mine + BLOCK, n - mine - BLOCK, lane);
        if (TOP) w.find_best(n - mine);
        else if (at == 0) w.template find_best<1>(n - mine);   // (enough to begin with)
        if (at == 0) w.start();
        if (TOP && at == 0) find_bound(qr_logit_key(w.largest));   // (the other waves add up in the meantime)
        w.template add<TOP>(n - mine);
        if (TOP && !over) {
            __syncthreads();
            if (VECTORS) w.vectors_to(vecs, index, &n_first, ROOM, least_of(shared_key), mine, lane);
            else w.hits(least_of(shared_key), x + mine, lane, [&](float f, int i) { push(qr_cand(qr_float_key(f + 0.0f), first + mine + i)); });
            if (more) {
                __syncthreads();
                const int count = n_first;
                over = count > ROOM;
                if (count > ROOM / 2 && !over) {   // uniform: what the list holds raises the bound and goes where it is below
                    QrChunk<T> held;   // (its first vectors)
                    int where[EACH];
                    QrCand c[EACH];
                    unsigned key[EACH], k = 0u;
#pragma unroll
                    for (int i = 0; i < EACH; ++i) {
                        key[i] = 0u;
                        const int from = tid + i * 64 * NW;
                        if (from >= count) continue;
                        if constexpr (VECTORS) {
                            held.raw[i] = vecs[from];
                            where[i] = index[from];
                            float f = held.at(i * V);
#pragma unroll
                            for (int j = 1; j < V; ++j) f = fmaxf(f, held.at(i * V + j));
                            key[i] = qr_logit_key(f);
                        } else {
                            c[i] = list[from];
                            key[i] = (unsigned)(c[i] >> 32);
                        }
                        k = key[i] > k ? key[i] : k;
                    }
                    find_bound(k);
                    if (tid == 0) n_first = 0;
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < EACH; ++i) {
                        if (key[i] == 0u || key[i] < shared_key) continue;
                        if constexpr (VECTORS) {
                            const int to = atomicAdd(&n_first, 1);
                            vecs[to] = held.raw[i];
                            index[to] = where[i];
                        } else {
                            push(c[i]);
                        }
                    }
                }
            }
        }
        if (!more) break;
        w.now = next;
    }
    const QrScoresSum own = w.sum();
    if (lane == 0) sums[wave] = own;
    __syncthreads();
    int M = 0;
    if (TOP) {
        M = n_first;
        over = M > ROOM;
        if (VECTORS && !over) {
            const float least = least_of(shared_key);
            for (int i = tid; i < M * V; i += 64 * NW) {
                const float f = (float)((const T *)pool)[i];
                if (f >= least) push(qr_cand(qr_float_key(f + 0.0f), first + index[i / V] + i % V));
            }
            __syncthreads();
            M = n_list;
            over = M > LIST;
        }
        if (over) {   // uniform
            __syncthreads();
            list[tid] = best_of_any<T, NW>(x, n, first, a.n, wave, lane, (QrLdsList)pool + wave * CAP);
            M = 64 * NW;
            __syncthreads();
        }
    }
    QrScoresSum sum = sums[lane & (NW - 1)];
    // (a wave whose r is above -MOST has one of its logits there; where all r are -MOST one such wave will do)
    if (__ballot(!sum.finite()) || !__ballot(sum.some())) {   // uniform
        __syncthreads();
        const QrScoresSum any = sums_of_any<T, NW>(x, n, wave, lane, most_of);
        if (lane == 0) sums[wave] = any;
        __syncthreads();
        sum = sums[lane & (NW - 1)];
    }
    QrScoresRow values;
    if (wave == 0) {   // joins the sums, the others rank
        double to = sum.r;
#pragma unroll
        for (int off = 1; off < NW; off <<= 1) to = fmax(to, __shfl_xor(to, off));
        sum.move(to);
#pragma unroll
        for (int off = 1; off < NW; off <<= 1) {
            sum.s += __shfl_xor(sum.s, off);
            sum.u += __shfl_xor(sum.u, off);
        }
        if (a.n_parts == 1) {
            values = QrScoresRow(sum);
            if (lane == 0) values.write(a, row, token);
        }
    } else if (TOP) {
        for (int i0 = 0; i0 < M; i0 += 16 * (NW - 1)) {   // uniform; four threads count for one candidate
            const int i = i0 + ((tid - 64) >> 2);
            const QrCand c = list[i < M ? i : 0];
            int rank = 0;
#pragma unroll 8
            for (int j = tid & 3; j < M; j += 4) rank += list[j] > c ? 1 : 0;
            rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, true);
            rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, true);
            if ((tid & 3) == 0 && i < M && c != 0ull && rank < a.n) ranked[rank] = c;
        }
    }
    const int64_t part = row * a.n_parts + blockIdx.x;
    if (a.n_parts > 1) {
        if (tid == 0) a.heads[part] = sum;
        if (TOP) {
            __syncthreads();
            if (tid < a.n) a.cands[part * a.n + tid] = ranked[tid];
        }
        return;
    }
    if (TOP) {
        __syncthreads();
        if (tid < a.n) values.write_rank(a, row, tid, ranked[tid]);   // (wave 0)
    }
}

// Rows that were cut: joins the parts' sums and lists.  Grid: one workgroup a row; a candidate to a thread.  Bound by latency: 3.9 us of the
// 15 of 64 x 131072 fp32 with 20 alternatives (4.7 before one wave joined the sums while the others rank).
template <class T>
__global__ __launch_bounds__(64 * MAX_PARTS) void scores_join_kernel(const QrScoresArgs a)
{
    __shared__ unsigned group_best[256];
    __shared__ QrCand all[64 * MAX_PARTS], ranked[MAX_TOP];
    __shared__ int n_all;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = blockIdx.x;
    QrCand mine = tid < a.n_parts * a.n ? a.cands[row * a.n_parts * a.n + tid] : 0ull;
    QrScoresToken token;
    QrScoresSum sum = {0.0, 0.0, 0.0};
    if (wave == 0) {
        token.load<T>(a, row);
        const int part = lane & (MAX_PARTS - 1);   // (every sixteen lanes do the same)
        if (part < a.n_parts) sum = a.heads[row * a.n_parts + part];
    }
    if (a.n > 0) {
        if (tid == 0) n_all = 0;
        if (tid < MAX_TOP) ranked[tid] = 0ull;
        unsigned bound = 1u;
        if (a.n_parts * a.n > 256) {   // (ranks of fewer are counted in less time than a bound takes)
            const unsigned four = qr_quad_max((unsigned)(mine >> 32));
            if ((lane & 3) == 0) group_best[tid >> 2] = four;
            __syncthreads();
            unsigned g[4], most = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                g[i] = group_best[i * 64 + lane];
                most = g[i] > most ? g[i] : most;
            }
            bound = qr_bound_of(g, qr_wave_reduce_u32<true>(most), a.n, a.n + a.n / 4);
        } else {
            __syncthreads();
        }
        if (mine != 0ull && (unsigned)(mine >> 32) >= bound) all[atomicAdd(&n_all, 1)] = mine;
        __syncthreads();
    }
    QrScoresRow values;
    if (wave == 0) {   // joins the sums, the others rank
        // (the r of a part that holds no finite logit, 0, may be above the others': it counts only where there is something to it)
        const bool some = sum.s != 0.0;
        double to = some ? sum.r : -1e300;
#pragma unroll
        for (int off = 1; off < MAX_PARTS; off <<= 1) to = fmax(to, __shfl_xor(to, off));
        if (some) sum.move(to);
        sum.r = to;
#pragma unroll
        for (int off = 1; off < MAX_PARTS; off <<= 1) {
            sum.s += __shfl_xor(sum.s, off);
            sum.u += __shfl_xor(sum.u, off);
        }
        values = QrScoresRow(sum);
        if (lane == 0) values.write(a, row, token);
    } else if (a.n > 0) {
        const int M = n_all;
        for (int i0 = 0; i0 < M; i0 += 16 * (MAX_PARTS - 1)) {   // uniform; four threads count for one candidate
            const int i = i0 + ((tid - 64) >> 2);
            const QrCand c = all[i < M ? i : 0];
            int rank = 0;
#pragma unroll 8
            for (int j = tid & 3; j < M; j += 4) rank += all[j] > c ? 1 : 0;
            rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, true);
            rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, true);
            if ((tid & 3) == 0 && i < M && rank < a.n) ranked[rank] = c;
        }
    }
    if (a.n > 0) {
        __syncthreads();
        if (tid < a.n) values.write_rank(a, row, tid, ranked[tid]);   // (wave 0)
    }
}

// Waves to a row, and parts of it.  A wave reads CHUNK = 256 vectors at a time, a workgroup of 16 waves 16 times as many.
// Measured (us; 1 / 4 / 8 / 16 waves), bf16, without alternatives: 4096 rows x 5000 10.3 / 10.7 / 14.6 / 23, 16384 x 8000 42 / 40 / 53 / 91, 16384 x
// 16000 101 / 97 / 87 / 116, 16384 x 32000 187 / 182 / 175 / 168, 4096 x 32000 41 / 42 / 42 / 39; with 5: 4096 x 5000 16.9 / 18.6 / 24 / 41, 16384 x
// 32000 219 / 247 / 230 / 261; with 16: 256 x 8000 12.5 / 5.9 / 5.5 / 6.2, 2048 x 5000 12.9 / 11.0 / 14.2 / 23, 4096 x 32000 66 / 64 / 53 / 67, 16384 x
// 8000 72 / 66 / 93 / 162, 16384 x 16000 127 / 133 / 123 / 200, 16384 x 32000 225 / 253 / 230 / 271; 256 x 131072 fp32 135 / 71 / 45 / 34.  In parts,
// with another launch that joins them (1 / 4 / 8 / 16 of them), fp32, 20 alternatives: 1 x 131072 20.0 / 10.4 / 8.5 / 8.6, 16 x 262144 40 / 19 / 12.7 /
// 10.7, 64 x 131072 34 / 13.2 / 12.7 / 17.1, 128 x 131072 36 / 22 / 20 / 27 (two 25); two pieces, 1 x 32000 with 5, 7.0 whole, 6.8 in four.
constexpr int FEW_ROWS = 256, STRETCH = 16384;   // (the shortest that a workgroup of 16 waves reads at a time)
void plan_scores(int rows, int V, int n, int chunk, int &waves, int &n_parts, int &part)
{
    const int chunks = (V + chunk - 1) / chunk;
    if (chunks == 1 || (chunks <= 3 && rows >= 2048 && n < 16) || (chunks > 8 && rows >= 8192 && n > 0)) waves = 1;
    else waves = chunks <= 6 ? 4 : chunks <= (n > 0 ? 24 : 15) ? 8 : 16;
    n_parts = 1;
    const int pieces = (chunks + 15) / 16;
    if (waves == 16 && pieces > 2 && rows < FEW_ROWS) {
        n_parts = pieces < FEW_ROWS / rows ? pieces : FEW_ROWS / rows;
        n_parts = n_parts < MAX_PARTS ? n_parts : MAX_PARTS;
    }
    part = qr_round_up((int)(((int64_t)V + n_parts - 1) / n_parts), 8);
    n_parts = (int)(((int64_t)V + part - 1) / part);
}
bool scores_sizes_ok(int32_t rows, int32_t V, int32_t n) { return rows >= 0 && V > 0 && n >= 0 && rows <= 1 << 25 && V <= 1 << 30 && n <= MAX_TOP; }
int most_parts(int32_t rows, int32_t V)   // of all rows together, of any call up to these sizes
{
    const int64_t each = ((int64_t)V + STRETCH - 1) / STRETCH, all = (each < MAX_PARTS ? each : MAX_PARTS) * rows;
    return (int)(all < FEW_ROWS ? all : FEW_ROWS);
}

template <class T, bool TOP>
void launch_scores(const QrScoresArgs &a, int waves, hipStream_t st)
{
    const int64_t n = waves == 1 ? ((int64_t)a.rows + 3) / 4 : a.rows;
    const dim3 grid(a.n_parts, (unsigned)(n < 32768 ? n : 32768), (unsigned)((n + 32767) / 32768));
    if (waves == 1) scores_wave_kernel<T, TOP><<<grid, 256, 0, st>>>(a);
    else if (waves == 4) scores_group_kernel<T, 4, TOP><<<grid, 256, 0, st>>>(a);
    else if (waves == 8) scores_group_kernel<T, 8, TOP><<<grid, 512, 0, st>>>(a);
    else scores_group_kernel<T, 16, TOP><<<grid, 1024, 0, st>>>(a);
    if (a.n_parts > 1) scores_join_kernel<T><<<a.rows, 64 * MAX_PARTS, 0, st>>>(a);
}

}  // namespace

extern "C" size_t qrnnt_token_scores_workspace(int32_t rows, int32_t V, int32_t n_top)
{
    if (!scores_sizes_ok(rows, V, n_top)) return 0;
    return (size_t)most_parts(rows, V) * (sizeof(QrScoresSum) + n_top * sizeof(QrCand)) + 256;
}

extern "C" qrnnt_status qrnnt_token_scores(const void *logits, int32_t dtype, int64_t ld, const int32_t *token, int32_t rows, int32_t V,
                                           int32_t n_top, float *logp_out, float *entropy_out, int32_t *top_token_out,
                                           float *top_logp_out, void *workspace, size_t workspace_bytes, void *stream)
{
    QR_REQUIRE(qr_is_dtype(dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(rows >= 0 && V > 0 && n_top >= 0 && ld >= V, QRNNT_ERR_SHAPE);
    QR_REQUIRE(scores_sizes_ok(rows, V, n_top) && qr_pitch_ok(rows, ld), QRNNT_ERR_UNSUPPORTED);
    if (rows == 0) return QRNNT_OK;
    QR_REQUIRE(logits && workspace && (token || !logp_out) && (n_top == 0 || (top_token_out && top_logp_out)), QRNNT_ERR_NULL);
    QR_REQUIRE(qr_aligned(logits, qr_dtype_size(dtype)) && qr_aligned(token, 4) && qr_aligned(logp_out, 4) && qr_aligned(entropy_out, 4) &&
                   qr_aligned(top_token_out, 4) && qr_aligned(top_logp_out, 4) && qr_aligned(workspace, 256), QRNNT_ERR_ALIGN);
    QR_REQUIRE(workspace_bytes >= qrnnt_token_scores_workspace(rows, V, n_top), QRNNT_ERR_WORKSPACE);
    QrScoresArgs a = {};
    a.logits = logits;  a.ld = ld;  a.token = token;  a.rows = rows;  a.V = V;  a.n = n_top;
    a.logp = logp_out;  a.entropy = entropy_out;  a.top_token = top_token_out;  a.top_logp = top_logp_out;
    int waves;
    plan_scores(rows, V, n_top, dtype == QRNNT_F32 ? QrChunk<float>::LEN : QrChunk<__bf16>::LEN, waves, a.n_parts, a.part);
    a.heads = (QrScoresSum *)workspace;
    a.cands = (QrCand *)((char *)workspace + (size_t)rows * a.n_parts * sizeof(QrScoresSum));
    auto launch = [&](auto zero) {
        using T = decltype(zero);
        if (n_top) launch_scores<T, true>(a, waves, (hipStream_t)stream);
        else launch_scores<T, false>(a, waves, (hipStream_t)stream);
    };
    if (dtype == QRNNT_F32) launch(0.0f);
    else if (dtype == QRNNT_F16) launch((_Float16)0.0f);
    else launch((__bf16)0.0f);
    return qr_launch_status();
}
