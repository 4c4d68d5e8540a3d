// Scores of given tokens, from logits: log probability of a row's token, entropy of the row, its best alternatives, in one pass
// over the logits.
//
// With S = sum exp(x - m), U = sum exp(x - m)(x - m) for any m:  lse = m + log S,  logp = (x[token] - m) - log S,
// entropy = log S - U / S.  Each lane keeps an m, S and U of what it has read (S and U in fp64) and joins them with the others' once, at
// the end of the row.  m is a logit that is at most LATE below the largest so far: sums move to another m seldom, and what they lose
// in moving (an exponential's rounding) weighs at most exp(-LATE) of them.
//
// The best alternatives: a wave knows a bound that n logits of the row reach; what reaches it goes to a list in LDS, out of which the
// n best are kept, and their smallest raises the bound, as often as the list fills.  The first bound is that of the groups of
// the wave's first logits.
#include <float.h>

#include "elem.h"
#include "kernels.h"
#include "select.h"

namespace {

constexpr int MAX_TOP = 64, CAP = 256;   // ranks; candidates in a wave's list
constexpr int MAX_PARTS = 16;

struct QrScoresHead {
    float top, pad;
    double s, u;
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
    QrScoresHead *heads;     // [rows][n_parts]
    QrCand *cands;           // [rows][n_parts][n], 0: none
};

constexpr float LOG2E = 1.4426950408889634f, FAR = -200.0f, LATE = 4.0f;   // exp(FAR) is 0 in fp32

// Sums relative to `top`, which starts at the lowest finite value: a row of nothing but -inf has S = 0.  NaN and +inf make S NaN.
struct QrScoresSum {
    float top = -FLT_MAX;
    double s = 0.0, u = 0.0;
    __device__ __forceinline__ QrScoresHead head() const { return {top, 0.0f, s, u}; }
    __device__ __forceinline__ void set(const QrScoresHead &h)
    {
        top = h.top;
        s = h.s;
        u = h.u;
    }
    // moves the sums to a top that is not below theirs
    __device__ __forceinline__ void move(float to)
    {
        const float d = fmaxf(top - to, FAR);
        const double c = (double)__builtin_amdgcn_exp2f(LOG2E * d);
        u = c * (u + (double)d * s);
        s *= c;
        top = to;
    }
    __device__ __forceinline__ void join_wave()
    {
        move(qr_key_float(qr_wave_reduce_u32<true>(qr_float_key(top))));
        s = qr_wave_sum(s);
        u = qr_wave_sum(u);
    }
};

// Value of a row's logits from its sums.
struct QrScoresRow {
    double top, log_s, entropy;
    bool none, bad;   // no token can be; a logit is NaN or +inf
    __device__ __forceinline__ explicit QrScoresRow(const QrScoresSum &a)
    {
        top = (double)a.top;
        none = a.s == 0.0;
        bad = !(a.s == a.s);
        log_s = log(a.s);
        entropy = none ? 0.0 : log_s - a.u / a.s;
    }
    __device__ __forceinline__ float logp(float logit) const { return none ? -INFINITY : (float)(((double)logit - top) - log_s); }
};

template <class T>
__device__ __forceinline__ void write_row(const QrScoresArgs &a, int64_t row, const QrScoresRow &r)
{
    if (a.logp) {
        const int t = a.token[row];
        a.logp[row] = t < 0 ? 0.0f : t >= a.V ? NAN : r.logp((float)((const T *)a.logits)[row * a.ld + t]);
    }
    if (a.entropy) a.entropy[row] = (float)r.entropy;
}
__device__ __forceinline__ void write_rank(const QrScoresArgs &a, int64_t row, int rank, QrCand c, const QrScoresRow &r)
{
    const bool some = c != 0ull && !r.bad;
    a.top_token[row * a.n + rank] = some ? qr_cand_index(c) : -1;
    a.top_logp[row * a.n + rank] = some ? r.logp(qr_cand_value(c)) : -INFINITY;
}

// Four vectors of a lane out of 256 that follow one another; -inf behind the end.
template <class T>
struct QrChunk {
    static constexpr int V = QrVec<T>::N, LEN = 256 * V, PER = 4 * V;
    typename QrVec<T>::type raw[4];
    __device__ __forceinline__ void load(const T *x, int n, int lane)
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int c = (v * 64 + lane) * V;
            if (c + V <= n) {
                raw[v] = *(const typename QrVec<T>::any *)(x + c);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) raw[v][i] = c + i < n ? x[c + i] : (T)-INFINITY;
            }
        }
    }
    __device__ __forceinline__ float at(int i) const { return (float)raw[i / V][i % V]; }
};

// A wave's list of candidates, in LDS; n and the bound are uniform.
struct QrTopList {
    QrCand *list;
    int count = 0;
    unsigned key = 0u;   // what is asked of a further candidate: a key not below this
    __device__ __forceinline__ float least() const { return key > 0x00800000u ? qr_key_float(key) : -FLT_MAX; }   // (keys up to there are those of -inf and below)

    // Keeps the n best, or up to `enough` while that needs no look at indices; returns the key that n of them reach (0: there are fewer).
    // (The bound is the n-th largest key itself unless no more than `enough` reach it: what is left is never more than that.)
    __device__ __forceinline__ unsigned keep_best(int n, int enough, int lane)
    {
        QrCand e[CAP / 64];
        unsigned g[CAP / 64], top = 0u;
#pragma unroll
        for (int j = 0; j < CAP / 64; ++j) {
            e[j] = lane + 64 * j < count ? list[lane + 64 * j] : 0ull;
            g[j] = (unsigned)(e[j] >> 32);
            top = g[j] > top ? g[j] : top;
        }
        const unsigned T = qr_bound_of(g, qr_wave_reduce_u32<true>(top), n, enough);
        if (T == 0u) return 0u;
        int above = 0, equal = 0;
#pragma unroll
        for (int j = 0; j < CAP / 64; ++j) {
            above += (int)__popcll(__ballot(g[j] > T));
            equal += (int)__popcll(__ballot(g[j] == T));
        }
        unsigned low = 0u;   // of the equal ones: the words (complements of the indices) from here on
        if (above + equal > enough) {
            for (int bit = 31; bit >= 0; --bit) {
                const unsigned trial = low | (1u << bit);
                int some = 0;
#pragma unroll
                for (int j = 0; j < CAP / 64; ++j) some += (int)__popcll(__ballot(g[j] == T && (unsigned)e[j] >= trial));
                if (above + some >= n) low = trial;
            }
        }
        int at = 0;
#pragma unroll
        for (int j = 0; j < CAP / 64; ++j) {
            const bool stays = g[j] > T || (g[j] == T && (unsigned)e[j] >= low);
            const unsigned long long m = __ballot(stays);
            if (stays) list[at + __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u))] = e[j];
            at += (int)__popcll(m);
        }
        count = at;
        __builtin_amdgcn_wave_barrier();
        return T;
    }
};

// Grid: x = part of a row, y (and z) = row, or four rows where a wave has one of its own (WPR 1).  WPR waves to a row.
template <class T, int WPR, bool TOP>
__global__ __launch_bounds__(WPR < 4 ? 256 : 64 * WPR) void scores_kernel(const QrScoresArgs a)
{
    constexpr int WAVES = WPR < 4 ? 4 : WPR, V = QrVec<T>::N, PER = QrChunk<T>::PER, LEN = QrChunk<T>::LEN;
    __shared__ QrCand lists[TOP ? WAVES : 1][TOP ? CAP : 1];
    __shared__ unsigned shared_key;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (WPR == 1) row = row * 4 + wave;
    const bool real = row < a.rows;   // uniform in a wave; of a workgroup with one row uniform at all
    if (!real) return;
    const int first = blockIdx.x * a.part, n = a.V - first < a.part ? a.V - first : a.part;
    const T *x = (const T *)a.logits + row * a.ld + first;
    QrTopList top;
    top.list = lists[TOP ? wave : 0];
    if (TOP && WPR > 1) {
        if (tid == 0) shared_key = 0u;
        __syncthreads();
    }
    QrScoresSum sum;
    QrChunk<T> now, next;
    const int at0 = (WPR == 1 ? 0 : wave) * LEN;
    if (at0 < n) now.load(x + at0, n - at0, lane);
    for (int at = at0; at < n; at += WPR * LEN) {
        const bool more = n - at > WPR * LEN;
        if (more) next.load(x + at + WPR * LEN, n - at - WPR * LEN, lane);
        float best[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            best[v] = now.at(v * V);
#pragma unroll
            for (int i = 1; i < V; ++i) best[v] = fmaxf(best[v], now.at(v * V + i));
        }
        const float largest = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
        const bool late = largest > sum.top + LATE;
        if (__ballot(late)) sum.move(late ? largest : sum.top);
        float s = 0.0f, u = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const float d = now.at(i) - sum.top, e = __builtin_amdgcn_exp2f(LOG2E * d);
            s += e;
            u = fmaf(e, fmaxf(d, FAR), u);
        }
        sum.s += (double)s;
        sum.u += (double)u;
        if (TOP) {
            if (at == at0) {
                unsigned g[4], most = 0u;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    g[v] = qr_logit_key(best[v]);
                    most = g[v] > most ? g[v] : most;
                }
                top.key = qr_bound_of(g, qr_wave_reduce_u32<true>(most), a.n, a.n + a.n / 4);
                if (WPR > 1 && lane == 0) atomicMax(&shared_key, top.key);
            }
            if (WPR > 1) {
                const unsigned k = __builtin_amdgcn_readfirstlane(*(volatile unsigned *)&shared_key);
                top.key = k > top.key ? k : top.key;
            }
            float least = top.least();
            if (__ballot(largest >= least)) {
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    if (!__ballot(best[v] >= least)) continue;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float f = now.at(v * V + i);
                        unsigned long long m = __ballot(f >= least);
                        if (!m) continue;
                        if (top.count + (int)__popcll(m) > CAP) {
                            // (n of the list reach the key, but what is left of these logits may lie in front of them)
                            const unsigned k = top.keep_best(a.n, a.n + a.n / 4, lane);
                            top.key = k > top.key ? k : top.key;
                            least = top.least();
                            m = __ballot(f >= least);
                        }
                        const int to = top.count + __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
                        if (f >= least) top.list[to] = qr_cand(qr_float_key(f + 0.0f), first + at + (v * 64 + lane) * V + i);
                        top.count += (int)__popcll(m);
                    }
                }
                __builtin_amdgcn_wave_barrier();
                if (top.count >= 2 * a.n + 16) {
                    const unsigned k = top.keep_best(a.n, a.n + a.n / 4, lane);
                    if (WPR > 1 && lane == 0) atomicMax(&shared_key, k);
                    // what this wave has not read yet lies behind: to be among the best it has to be larger
                    top.key = k + 1u > top.key ? k + 1u : top.key;
                }
            }
        }
        if (more) now = next;
    }
    sum.join_wave();
    if (TOP && top.count > a.n) top.keep_best(a.n, a.n, lane);
    QrCand mine = TOP && lane < top.count ? top.list[lane] : 0ull;
    if (WPR == 1) {
        const QrScoresRow r(sum);
        if (lane == 0) write_row<T>(a, row, r);
        if (TOP) {
            int rank = 0;
            for (int j = 0; j < top.count; ++j) rank += top.list[j] > mine ? 1 : 0;
            if (lane < a.n) write_rank(a, row, lane < top.count ? rank : lane, mine, r);
        }
        return;
    }
    // the waves' sums and lists
    __shared__ QrScoresHead sums[WAVES];
    __shared__ unsigned group_best[256];
    __shared__ QrCand all[TOP ? 64 * WAVES : 1];
    __shared__ int n_all;
    if (lane == 0) sums[wave] = sum.head();
    if (TOP) {
        if (tid == 0) n_all = 0;
        const unsigned k = (unsigned)(mine >> 32);
        if (WAVES == 4) {
            group_best[tid] = k;
        } else {
            const unsigned four = qr_quad_max(k);
            if ((lane & 3) == 0) group_best[tid >> 2] = four;
        }
    }
    __syncthreads();
    sum = QrScoresSum();
    if (lane < WAVES) sum.set(sums[lane]);
    sum.join_wave();
    const int64_t part = row * a.n_parts + blockIdx.x;
    if (TOP) {
        unsigned g[4], most = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            g[i] = group_best[i * 64 + lane];
            most = g[i] > most ? g[i] : most;
        }
        const unsigned bound = qr_bound_of(g, qr_wave_reduce_u32<true>(most), a.n, a.n + a.n / 4);
        if (mine != 0ull && (unsigned)(mine >> 32) >= bound) all[atomicAdd(&n_all, 1)] = mine;
        __syncthreads();
    }
    const QrScoresRow r(sum);
    if (tid == 0) {
        if (a.n_parts > 1) a.heads[part] = sum.head();
        else write_row<T>(a, row, r);
    }
    if (TOP) {
        const int M = n_all;
        auto put = [&](int rank, QrCand c) {
            if (a.n_parts > 1) a.cands[part * a.n + rank] = c;
            else write_rank(a, row, rank, c, r);
        };
        for (int i0 = 0; i0 < M; i0 += 16 * WAVES) {   // uniform; four threads count for one candidate
            const int i = i0 + (tid >> 2);
            const QrCand c = all[i < M ? i : 0];
            int rank = 0;
            for (int j = tid & 3; j < M; j += 4) rank += all[j] > c ? 1 : 0;
            rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, true);
            rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, true);
            if ((tid & 3) == 0 && i < M && rank < a.n) put(rank, c);
        }
        if (tid >= M && tid < a.n) put(tid, 0ull);
    }
}

// Rows that were cut: joins the parts' sums and lists.  Grid: one workgroup a row; a candidate to a thread.
template <class T>
__global__ __launch_bounds__(64 * MAX_PARTS) void scores_join_kernel(const QrScoresArgs a)
{
    __shared__ unsigned group_best[256];
    __shared__ QrCand all[64 * MAX_PARTS];
    __shared__ int n_all;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    QrCand mine = tid < a.n_parts * a.n ? a.cands[row * a.n_parts * a.n + tid] : 0ull;
    QrScoresSum sum;
    if (lane < a.n_parts) sum.set(a.heads[row * a.n_parts + lane]);
    sum.join_wave();
    const QrScoresRow r(sum);
    if (tid == 0) {
        n_all = 0;
        write_row<T>(a, row, r);
    }
    if (a.n == 0) return;
    const unsigned four = qr_quad_max((unsigned)(mine >> 32));
    if ((lane & 3) == 0) group_best[tid >> 2] = four;
    __syncthreads();
    unsigned g[4], most = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = group_best[i * 64 + lane];
        most = g[i] > most ? g[i] : most;
    }
    const unsigned bound = qr_bound_of(g, qr_wave_reduce_u32<true>(most), a.n, a.n + a.n / 4);
    if (mine != 0ull && (unsigned)(mine >> 32) >= bound) all[atomicAdd(&n_all, 1)] = mine;
    __syncthreads();
    const int M = n_all;
    for (int i0 = 0; i0 < M; i0 += 16 * MAX_PARTS) {   // uniform
        const int i = i0 + (tid >> 2);
        const QrCand c = all[i < M ? i : 0];
        int rank = 0;
        for (int j = tid & 3; j < M; j += 4) rank += all[j] > c ? 1 : 0;
        rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, true);
        rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, true);
        if ((tid & 3) == 0 && i < M && rank < a.n) write_rank(a, row, rank, c, r);
    }
    if (tid >= M && tid < a.n) write_rank(a, row, tid, 0ull, r);
}

// Waves to a row, and parts of it.
constexpr int FEW_ROWS = 256, STRETCH = 16384;
void plan_scores(int rows, int V, int &waves, int &n_parts, int &part)
{
    waves = rows >= 4096 || V <= 2048 ? 1 : rows >= 1024 || V <= 8192 ? 4 : 16;
    n_parts = 1;
    if (waves == 16 && rows < FEW_ROWS) {
        n_parts = (V + STRETCH - 1) / STRETCH;
        n_parts = n_parts < FEW_ROWS / rows ? n_parts : FEW_ROWS / rows;
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
    if (waves == 1) scores_kernel<T, 1, TOP><<<grid, 256, 0, st>>>(a);
    else if (waves == 4) scores_kernel<T, 4, TOP><<<grid, 256, 0, st>>>(a);
    else scores_kernel<T, 16, TOP><<<grid, 1024, 0, st>>>(a);
    if (a.n_parts > 1) scores_join_kernel<T><<<a.rows, 64 * MAX_PARTS, 0, st>>>(a);
}

}  // namespace

extern "C" size_t qrnnt_token_scores_workspace(int32_t rows, int32_t V, int32_t n_top)
{
    if (!scores_sizes_ok(rows, V, n_top)) return 0;
    return (size_t)most_parts(rows, V) * (sizeof(QrScoresHead) + n_top * sizeof(QrCand)) + 256;
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
    plan_scores(rows, V, waves, a.n_parts, a.part);
    a.heads = (QrScoresHead *)workspace;
    a.cands = (QrCand *)((char *)workspace + (size_t)rows * a.n_parts * sizeof(QrScoresHead));
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
