// Beam selection over large vocabularies, from logits: log-softmax, scores and the best extensions of a beam (Sec. 2: up
// to W hypotheses are kept per iteration) in one pass over the logits.
//
// A hypothesis' candidates are ordered as its logits are, so a stretch of a row can give up all but its n_out largest
// logits before the row's log-sum-exp is known.  First launch: one workgroup per stretch holds it in registers, finds its
// maximum, sum of exponentials and n_out largest logits.  Second launch: one workgroup per utterance joins sums and lists.
#include "elem.h"
#include "kernels.h"
#include "select.h"

namespace {

constexpr int MAX_OUT = 64;      // ranks
constexpr int LIST = 512;        // candidates that a selection holds in LDS (more: it goes rank by rank)

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
    struct QrPartHead *heads;    // [B*W][n_parts]
    QrCand *cands;               // [B*W][n_parts][K]: (key of the logit, token), best first, 0: none
};

struct QrPartHead {
    float top, pad;              // the stretch's largest logit (-inf: none)
    double sum;                  // sum of exp(logit - top); NaN where a logit is NaN or +inf
};

__device__ __forceinline__ bool takes_part(const QrSelectArgs &a, int64_t row)
{
    const float s = a.score[row];
    return s > -INFINITY && !(a.finished && a.finished[row]);
}

// Grid: x = stretch, y (and z) = row.  256 threads, NV vectors of 16 bytes each.
template <class T, int NV>
__global__ __launch_bounds__(256) void select_parts_kernel(const QrSelectArgs a)
{
    constexpr int V = QrVec<T>::N, PER = NV * V;
    __shared__ QrCand list[LIST], best[MAX_OUT], wave_best[4];
    __shared__ unsigned group_best[256];
    __shared__ double wave_sum[4];
    __shared__ int n_list;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= (int64_t)a.B * a.W || !takes_part(a, row)) return;   // uniform; the second launch does not ask for it either
    const int first = blockIdx.x * a.part, n = a.V - first < a.part ? a.V - first : a.part;
    const T *x = (const T *)a.logits + row * a.ld + first;
    if (tid == 0) n_list = 0;
    if (tid < MAX_OUT) best[tid] = 0;
    float f[PER];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float u[V];
        const int c = (v * 256 + tid) * V;
        if (c + V <= n) {
            qr_load_vec(x + c, u);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] = c + i < n ? (float)x[c + i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) f[v * V + i] = u[i];
    }
    float largest = -INFINITY;   // (NaN is passed over here and found again in the sum)
#pragma unroll
    for (int i = 0; i < PER; ++i) largest = fmaxf(largest, f[i]);
    group_best[tid] = largest > -INFINITY ? qr_float_key(largest + 0.0f) : 0u;
    __syncthreads();
    unsigned g[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = group_best[i * 64 + lane];
    const QrBound bound(g, a.K);
    const float top = bound.top ? bound.v_max : -INFINITY;
    if (a.log_softmax) {
        const float m = bound.top ? top : 0.0f;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) s += qr_exp(f[i] - m);
        double d = (double)s;
        for (int off = 32; off > 0; off >>= 1) d += __shfl_xor(d, off);
        if (lane == 0) wave_sum[wave] = d;
    }
    auto cand = [&](int i) -> QrCand {
        return f[i] > -INFINITY ? qr_cand(qr_float_key(f[i] + 0.0f), first + ((i / V) * 256 + tid) * V + i % V) : 0ull;
    };
    // what passes the bound goes to the list
    int n_pass = 0;
    bool in[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        in[i] = f[i] > -INFINITY && bound.passes(qr_float_key(f[i] + 0.0f));
        n_pass += in[i] ? 1 : 0;
    }
    if (n_pass) {
        int pos = atomicAdd(&n_list, n_pass);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (in[i] && pos < LIST) list[pos++] = cand(i);
    }
    __syncthreads();
    if (n_list <= LIST) {
        qr_rank(list, n_list, a.K, tid, best);
    } else {   // many equal logits: rank by rank over what the threads hold
        QrCand last = ~0ull;
        for (int r = 0; r < a.K; ++r) {
            QrCand mine = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const QrCand c = cand(i);
                if (c < last && c > mine) mine = c;
            }
            for (int off = 32; off > 0; off >>= 1) {
                const QrCand o = __shfl_xor(mine, off);
                mine = o > mine ? o : mine;
            }
            if (lane == 0) wave_best[wave] = mine;
            __syncthreads();
            for (int w = 0; w < 4; ++w) mine = wave_best[w] > mine ? wave_best[w] : mine;
            __syncthreads();
            if (tid == 0) best[r] = mine;
            last = mine;   // 0: nothing is smaller, the ranks that follow stay empty
        }
    }
    __syncthreads();
    const int64_t part = row * a.n_parts + blockIdx.x;
    if (tid < a.K) a.cands[part * a.K + tid] = best[tid];
    if (tid == 0) a.heads[part] = {top, 0.0f, a.log_softmax ? wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3] : 0.0};
}

// Values of the whole beam's candidates as words.
__device__ __forceinline__ unsigned long long order_of(double v)   // larger double <=> larger word; 0 for what is never taken
{
    if (!(v > -INFINITY)) return 0ull;
    const unsigned long long u = __double_as_longlong(v + 0.0);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(unsigned long long o)
{
    return __longlong_as_double((o >> 63) ? (o & 0x7FFFFFFFFFFFFFFFull) : ~o);
}

// Grid: one workgroup an utterance.
__global__ __launch_bounds__(256) void select_beam_kernel(const QrSelectArgs a)
{
    __shared__ unsigned long long l_val[LIST], l_cand[LIST];   // value; (logit, token)
    __shared__ int l_hyp[LIST];
    __shared__ unsigned group_best[256];
    // logit - lse = (logit - top) - log(sum of exp(logit - top)): with the two apart also logits of the type's lowest value, next
    // to which the logarithm vanishes, give what they mean.  log_sum NaN: no candidates.
    __shared__ double row_top[64], log_sum[64];
    __shared__ int n_list;
    __shared__ unsigned long long r_val[4], r_cand[4];
    __shared__ int r_hyp[4];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = (int64_t)b * a.W;
    const int per = a.n_parts * a.K;
    if (tid == 0) n_list = 0;
    if (tid < a.W) {
        const int64_t row = row0 + tid;
        double ls = NAN;
        float top = -INFINITY;
        if (takes_part(a, row)) {
            const QrPartHead *h = a.heads + row * a.n_parts;
            ls = 0.0;
            if (a.log_softmax) {
                for (int i = 0; i < a.n_parts; ++i) top = fmaxf(top, h[i].top);
                for (int i = 0; i < a.n_parts; ++i) ls += h[i].sum * exp((double)h[i].top - (double)top);   // (of -inf alone: NaN)
                ls = log(ls);
            }
        }
        row_top[tid] = a.log_softmax ? (double)top : 0.0;
        log_sum[tid] = ls;
    }
    __syncthreads();
    auto value = [&](int w, QrCand c) -> double {
        return c == 0 ? -INFINITY : (double)a.score[row0 + w] + (((double)qr_cand_value(c) - row_top[w]) - log_sum[w]);
    };
    // every candidate of the beam: visit(value order, (logit, token), hypothesis)
    auto each = [&](auto &&visit) {
        for (int i = tid; i < a.W * per; i += 256) {
            const int w = i / per;
            if (log_sum[w] == log_sum[w]) {
                const QrCand c = a.cands[row0 * per + i];
                const unsigned long long o = order_of(value(w, c));
                if (o) visit(o, c, w);
            }
        }
        if (a.finished && tid < a.W && a.finished[row0 + tid]) {
            const unsigned long long o = order_of((double)a.score[row0 + tid]);
            if (o) visit(o, qr_cand(1u, a.end_token), tid);
        }
    };
    unsigned top = 0u;
    each([&](unsigned long long o, QrCand, int) { const unsigned k = (unsigned)(o >> 32); top = k > top ? k : top; });
    group_best[tid] = top;
    __syncthreads();
    // the K-th largest of the 256 threads' best is a bound from below of the K-th best (upper 32 bits of the order)
    unsigned g[4], T = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = group_best[i * 64 + lane];
    for (int bit = 31; bit >= 0; --bit) {
        const unsigned trial = T | (1u << bit);
        int cnt = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) cnt += (int)__popcll(__ballot(g[i] >= trial));
        if (cnt >= a.K) T = trial;
        if (cnt == a.K) break;
    }
    each([&](unsigned long long o, QrCand c, int w) {
        if ((unsigned)(o >> 32) >= T) {
            const int at = atomicAdd(&n_list, 1);
            if (at < LIST) { l_val[at] = o; l_cand[at] = c; l_hyp[at] = w; }
        }
    });
    __syncthreads();
    const int64_t out0 = (int64_t)b * a.K;
    auto put = [&](int r, unsigned long long o, QrCand c, int w) {
        a.parent_out[out0 + r] = o ? w : -1;
        a.token_out[out0 + r] = o ? qr_cand_index(c) : -1;
        a.score_out[out0 + r] = o ? (float)value_of(o) : -INFINITY;
        if (a.finished_out) a.finished_out[out0 + r] = o && ((a.finished && a.finished[row0 + w]) || qr_cand_index(c) == a.end_token) ? 1 : 0;
    };
    auto better = [](unsigned long long o, QrCand c, int w, unsigned long long o2, QrCand c2, int w2) {
        return o != o2 ? o > o2 : (w != w2 ? w < w2 : c > c2);
    };
    if (n_list <= LIST) {
        const int M = n_list;
        for (int i = tid; i < M; i += 256) {
            const unsigned long long o = l_val[i], c = l_cand[i];
            const int w = l_hyp[i];
            int rank = 0;
            for (int j = 0; j < M; ++j) rank += better(l_val[j], l_cand[j], l_hyp[j], o, c, w) ? 1 : 0;
            if (rank < a.K) put(rank, o, c, w);
        }
        for (int r = M + tid; r < a.K; r += 256) put(r, 0ull, 0ull, 0);
        return;
    }
    // many equal values: rank by rank
    unsigned long long last_o = ~0ull, last_c = ~0ull;
    int last_w = -1;
    for (int r = 0; r < a.K; ++r) {
        unsigned long long bo = 0, bc = 0;
        int bw = 0x7fffffff;
        each([&](unsigned long long o, QrCand c, int w) {
            if (better(last_o, last_c, last_w, o, c, w) && better(o, c, w, bo, bc, bw)) { bo = o; bc = c; bw = w; }
        });
        for (int off = 32; off > 0; off >>= 1) {
            const unsigned long long o = __shfl_xor(bo, off), c = __shfl_xor(bc, off);
            const int w = __shfl_xor(bw, off);
            if (better(o, c, w, bo, bc, bw)) { bo = o; bc = c; bw = w; }
        }
        if (lane == 0) { r_val[wave] = bo; r_cand[wave] = bc; r_hyp[wave] = bw; }
        __syncthreads();
        for (int i = 0; i < 4; ++i)
            if (better(r_val[i], r_cand[i], r_hyp[i], bo, bc, bw)) { bo = r_val[i]; bc = r_cand[i]; bw = r_hyp[i]; }
        __syncthreads();
        if (tid == 0) put(r, bo, bc, bw);
        last_o = bo;
        last_c = bc;
        last_w = bw;
    }
}

// How a row is cut: stretches of at most 8192 logits, shorter ones where there are few rows.
void plan_select(int64_t rows, int V, int &n_parts, int &part)
{
    const int len = rows * ((V + 8191) / 8192) >= 256 ? 8192 : 2048;
    n_parts = (V + len - 1) / len;
    part = qr_round_up((V + n_parts - 1) / n_parts, 8);
    n_parts = (V + part - 1) / part;
}

bool select_sizes_ok(int32_t B, int32_t W, int32_t V, int32_t K)
{
    return B >= 0 && W > 0 && V > 0 && K > 0 && W <= 64 && K <= MAX_OUT && (int64_t)W * V <= INT32_MAX && (int64_t)B * W <= INT32_MAX;
}

size_t heads_bytes(int64_t rows, int n_parts) { return ((size_t)rows * n_parts * sizeof(QrPartHead) + 255) / 256 * 256; }

template <class T>
void launch_parts(const QrSelectArgs &a, hipStream_t st)
{
    const int64_t rows = (int64_t)a.B * a.W;
    const dim3 grid(a.n_parts, (unsigned)(rows < 32768 ? rows : 32768), (unsigned)((rows + 32767) / 32768));
    constexpr int V = QrVec<T>::N;
    if (a.part <= 2048) select_parts_kernel<T, 2048 / 256 / V><<<grid, 256, 0, st>>>(a);
    else select_parts_kernel<T, 8192 / 256 / V><<<grid, 256, 0, st>>>(a);
}

}  // namespace

extern "C" size_t qrnnt_beam_select_workspace(int32_t B, int32_t W, int32_t V, int32_t n_out)
{
    if (!select_sizes_ok(B, W, V, n_out)) return 0;
    int n_parts, part;
    const int64_t rows = (int64_t)(B > 0 ? B : 1) * W;
    plan_select(rows, V, n_parts, part);
    return heads_bytes(rows, n_parts) + (size_t)rows * n_parts * n_out * sizeof(QrCand);
}

extern "C" qrnnt_status qrnnt_beam_select(const float *score, const void *logits, int32_t dtype, int64_t ld, int32_t log_softmax,
                                          const uint8_t *finished, int32_t end_token, int32_t B, int32_t W, int32_t V,
                                          int32_t n_out, int32_t *parent_out, int32_t *token_out, float *score_out,
                                          uint8_t *finished_out, void *workspace, size_t workspace_bytes, void *stream)
{
    QR_REQUIRE(qr_is_dtype(dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(B >= 0 && W > 0 && V > 0 && n_out > 0 && ld >= V, QRNNT_ERR_SHAPE);
    QR_REQUIRE(select_sizes_ok(B, W, V, n_out), QRNNT_ERR_UNSUPPORTED);
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
    const int64_t rows = (int64_t)B * W;
    plan_select(rows, V, a.n_parts, a.part);
    a.heads = (QrPartHead *)workspace;
    a.cands = (QrCand *)((char *)workspace + heads_bytes(rows, a.n_parts));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == QRNNT_F32) launch_parts<float>(a, st);
    else if (dtype == QRNNT_F16) launch_parts<_Float16>(a, st);
    else launch_parts<__bf16>(a, st);
    select_beam_kernel<<<B, 256, 0, st>>>(a);
    return qr_launch_status();
}
