// 8-bit activations with a range for each row: the MAX range picker of Sec. 3.1 on activations, by itself
// (qrnnt_quantize_tokens) and behind a residual sum and a root-mean-square norm (qrnnt_rms_norm_quant).
//
// q = rne(127 u / max|u|) with u = h * weight: the root mean square of the row divides u and its range alike, so the codes
// need the largest |u| only and the root enters the scale.  One pass over memory: a row's u stay in registers between
// the reduction and the codes.
#include "elem.h"
#include "kernels.h"

namespace {

struct QrTokenArgs {
    const void *x, *residual, *weight;
    void *sum;
    int64_t rows, ld_x, ld_res, ld_sum;
    int cols, ld_q;
    float eps;
    int8_t *q;
    float *scale;
};

// What a row reduces to.  key: largest |u| as bits (NaN above infinity above numbers).  peak: the largest |u| where fp32
// does not hold the products exactly.
template <bool WIDE>
struct QrRowSums {
    float ss;
    unsigned key;
    double peak;

    __device__ __forceinline__ void add(const QrRowSums &o)
    {
        ss += o.ss;
        key = o.key > key ? o.key : key;
        if (WIDE) peak = fmax(peak, o.peak);
    }
    // Over LANES neighbouring lanes (the row's, or the wave's).
    template <int LANES>
    __device__ __forceinline__ void reduce_wave(bool sums)
    {
        if (sums)
            for (int off = LANES / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        if (LANES == 64) {
            key = qr_wave_reduce_u32<true>(key);
        } else {
            for (int off = LANES / 2; off > 0; off >>= 1) {
                const unsigned o = __shfl_xor(key, off);
                key = o > key ? o : key;
            }
        }
        if (WIDE)
            for (int off = LANES / 2; off > 0; off >>= 1) peak = fmax(peak, __shfl_xor(peak, off));
    }
};

// Sum, largest value and "all finite" over the threads of a row, in fp64 (rows out of fp32's comfort only).
template <int TPR>
__device__ __forceinline__ void reduce_row64(double &sum, double &peak, bool &bad, double *lds)
{
    int any_bad = bad ? 1 : 0;
    for (int off = (TPR < 64 ? TPR : 64) / 2; off > 0; off >>= 1) {
        sum += __shfl_xor(sum, off);
        peak = fmax(peak, __shfl_xor(peak, off));
        any_bad |= __shfl_xor(any_bad, off);
    }
    bad = any_bad != 0;
    if (TPR > 64) {
        constexpr int NW = TPR / 64;
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            lds[wave] = sum;
            lds[NW + wave] = peak;
            lds[2 * NW + wave] = bad ? 1.0 : 0.0;
        }
        __syncthreads();
        sum = 0.0, peak = 0.0;
        double any = 0.0;
        for (int w = 0; w < NW; ++w) {
            sum += lds[w];
            peak = fmax(peak, lds[NW + w]);
            any += lds[2 * NW + w];
        }
        bad = any != 0.0;
    }
}

// rne(127 u / peak).  WIDE: u and peak are products of two fp32 values, whose 127-fold (55 bits) fp64 does not hold; where the quotient is next
// to the border of two codes the sign of 254 u - (2 j + 1) peak decides, each product as its rounded value and the rest of it.  (Otherwise u
// and peak have at most 24 bits, and what is not at a border is further from it than 2^-32 of the quotient.)
template <bool WIDE>
__device__ __forceinline__ int code_of(double u, double peak)
{
    const double q = 127.0 * u / peak;
    int k = (int)rint(q);
    if (WIDE && fabs(fabs(q - k) - 0.5) < 0x1p-40) {
        const double j = floor(q), a = 254.0 * u, m = 2.0 * j + 1.0, b = m * peak;
        const double d = (a - b) + (fma(254.0, u, -a) - fma(m, peak, -b));
        k = (int)j + (d > 0.0 || (d == 0.0 && ((int)j & 1)) ? 1 : 0);
    }
    return k;
}

// A row whose values fp32 does not carry well: all zero, not finite, squares or products that overflow or vanish.  All
// of it in fp64, from the stored h.
template <class T, bool NORM, int TPR>
__device__ __forceinline__ void odd_row(const T *h, const T *weight, int cols, float eps, int t, int8_t *q, float *scale, double *lds)
{
    constexpr int V = QrVec<T>::N;
    double sum = 0.0, peak = 0.0;
    bool bad = false;
    auto value = [&](int c) { return (double)(float)h[c] * (NORM && weight ? (double)(float)weight[c] : 1.0); };
    for (int c0 = t * V; c0 < cols; c0 += TPR * V)
        for (int i = 0; i < V && c0 + i < cols; ++i) {
            const double u = value(c0 + i), hd = (double)(float)h[c0 + i];
            bad |= !(fabs(u) < INFINITY) || !(fabs(hd) < INFINITY);
            peak = fmax(peak, fabs(u));
            sum += hd * hd;
        }
    reduce_row64<TPR>(sum, peak, bad, lds);
    const bool none = bad || peak == 0.0;
    for (int c0 = t * V; c0 < cols; c0 += TPR * V)
        for (int i = 0; i < V && c0 + i < cols; ++i) q[c0 + i] = none ? 0 : (int8_t)code_of<NORM && sizeof(T) == 4>(value(c0 + i), peak);
    if (t == 0) {
        const double root = NORM ? sqrt(sum / cols + (double)eps) : 1.0;
        *scale = bad ? NAN : (peak == 0.0 ? 1.0f : (float)(peak / root / 127.0));
    }
}

// Bound by memory: 16384 x 4096 bf16 with residual, 470 MB, in 83 us where calls follow one another is 5.6 TB/s (a copy of 1 GiB on this
// card: 5.2), and 92 in the trace of a program that multiplies codes and scales in between; fp32, 872 MB, 146.  One row of 4096 takes 4
// us, the length of its chain.
// TPR threads to a row (up to 64: workgroups of 256 have several), PER vectors of 16 bytes to a thread; PER = 0: rows of any length, read
// a second time for the codes.
template <class T, bool NORM, int TPR, int PER>
__global__ __launch_bounds__(TPR < 128 ? 256 : TPR) void tokens_kernel(const QrTokenArgs a)
{
    constexpr int V = QrVec<T>::N, RPB = TPR < 128 ? 256 / TPR : 1, NW = TPR < 64 ? 1 : TPR / 64;
    constexpr bool WIDE = NORM && sizeof(T) == 4;   // products of two fp32 values do not fit fp32
    __shared__ QrRowSums<WIDE> red[NW > 1 ? NW : 1];
    __shared__ double red64[3 * NW];
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= a.rows) return;   // (where rows share a workgroup nothing waits for others)
    const int t = threadIdx.x % TPR, cols = a.cols;
    const T *x = (const T *)a.x + row * a.ld_x, *res = (const T *)a.residual, *weight = (const T *)a.weight;
    T *sum = (T *)a.sum;
    if (NORM && res) {
        res += row * a.ld_res;
        sum += row * a.ld_sum;
    }
    const T *h_at = NORM && res ? sum : x;   // where h can be read again
    int8_t *q = a.q + row * a.ld_q;

    QrRowSums<WIDE> s = {0.0f, 0u, 0.0};
    // h of the vector at column c from its inputs; stores the sum
    auto form = [&](int c, float (&v)[V], const float (&r)[V]) {
        if (NORM && res) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = (float)(T)(v[i] + r[i]);
            qr_store_vec(sum + c, cols - c, v);
        }
    };
    // v: h on entry, u on return
    auto take = [&](float (&v)[V], const float (&w)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (NORM) s.ss = fmaf(v[i], v[i], s.ss);
            if (WIDE) s.peak = fmax(s.peak, fabs((double)v[i] * (double)w[i]));
            if (NORM) v[i] *= w[i];
            const unsigned k = __float_as_uint(v[i]) & 0x7FFFFFFFu;
            s.key = k > s.key ? k : s.key;
        }
    };
    auto ones = [](float (&w)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = 1.0f;
    };

    constexpr int P = PER ? PER : 1;
    float u[P][V];
    if (PER) {
        // all loads of the row first: a vector that lies inside the row as it is, what hangs over its end element by element
        float r[P][V], w[P][V];
        const int t_wave = __builtin_amdgcn_readfirstlane(t & ~63);
        // None of the wave's vectors is in the row (uniform): not computed.  (fp32 without a norm has so little to compute that the
        // branches between its loads cost more: 16384 x 1100 16.2 us, with them 17.9; bf16 with residual, 608 columns 27.1 and 25.0.)
        auto idle = [&](int p) { return (NORM || sizeof(T) == 2) && (p * TPR + t_wave) * V >= cols; };
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (idle(p)) continue;
            const int c = (p * TPR + t) * V, n = cols - c;
            const bool whole = n >= V;
            if (cols >= V) {   // uniform
                const int at = whole ? c : 0;
                qr_load_vec(x + at, u[p]);
                if (NORM && res) qr_load_vec(res + at, r[p]);
                if (NORM && weight) qr_load_vec(weight + at, w[p]);
            }
            if (!whole) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    u[p][i] = i < n ? (float)x[c + i] : 0.0f;
                    if (NORM && res) r[p][i] = i < n ? (float)res[c + i] : 0.0f;
                    if (NORM && weight) w[p][i] = i < n ? (float)weight[c + i] : 0.0f;
                }
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (idle(p)) continue;
            const int c = (p * TPR + t) * V;
            if (!(NORM && weight)) ones(w[p]);
            form(c, u[p], r[p]);
            take(u[p], w[p]);
        }
    } else {
        double ss = 0.0;   // (a thread adds up any number of vectors)
        for (int c = t * V; c < cols; c += TPR * V) {
            float r[V], w[V];
            qr_load_vec(x + c, cols - c, 0.0f, u[0]);
            if (NORM && res) qr_load_vec(res + c, cols - c, 0.0f, r);
            if (NORM && weight) qr_load_vec(weight + c, cols - c, 0.0f, w);
            else ones(w);
            form(c, u[0], r);
            take(u[0], w);
            ss += (double)s.ss;
            s.ss = 0.0f;
        }
        s.ss = (float)ss;
    }
    s.template reduce_wave<(TPR < 64 ? TPR : 64)>(NORM);
    if (NW > 1) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
        __syncthreads();
        s = red[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) s.add(red[w]);
    }
    const float peak = WIDE ? (float)s.peak : __uint_as_float(s.key);
    // padding behind the last vector: up to 15 bytes, in words
    if (t < 3 && qr_round_up(cols, V) + 4 * t < qr_act_pitch(cols)) *(unsigned *)(q + qr_round_up(cols, V) + 4 * t) = 0u;
    if (!(peak >= 0x1p-60f && peak <= 0x1p100f && s.key < 0x7F800000u && (!NORM || (s.ss >= 0x1p-80f && s.ss < INFINITY)))) {   // uniform over the row
        if (t < V && cols + t < qr_round_up(cols, V)) q[cols + t] = 0;
        odd_row<T, NORM, TPR>(h_at, weight, cols, a.eps, t, q, a.scale + row, red64);
        return;
    }
    const float inv = 127.0f / peak;
    // u * inv is off by at most 4 roundings of 127 (3.1e-5; of u and peak where they are products of fp32 values, of inv, of this product):
    // where it is nearer than 2^-14 (6.1e-5) to the border of two codes the quotient itself decides
    auto codes = [&](int c, const float (&v)[V]) {
        int k[V];
        bool near = false;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float p = v[i] * inv, r = __builtin_rintf(p);
            near |= fabsf(p - r) > 0.5f - 0x1p-14f;
            k[i] = (int)r;
        }
        if (near) {
            const double pk = WIDE ? s.peak : (double)peak;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                double e = (double)v[i];
                if (WIDE && c + i < cols) e = (double)(float)h_at[c + i] * (weight ? (double)(float)weight[c + i] : 1.0);
                k[i] = code_of<WIDE>(e, pk);
            }
        }
#pragma unroll
        for (int i = 0; i < V; i += 4)
            *(unsigned *)(q + c + i) = (unsigned)(k[i] & 0xFF) | (unsigned)(k[i + 1] & 0xFF) << 8 | (unsigned)(k[i + 2] & 0xFF) << 16 | (unsigned)k[i + 3] << 24;
    };
    if (PER) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (p * TPR + t) * V;
            if (c < cols) codes(c, u[p]);
        }
    } else {
        for (int c = t * V; c < cols; c += TPR * V) {
            float w[V];
            qr_load_vec(h_at + c, cols - c, 0.0f, u[0]);
            if (NORM && weight) {
                qr_load_vec(weight + c, cols - c, 0.0f, w);
#pragma unroll
                for (int i = 0; i < V; ++i) u[0][i] *= w[i];
            }
            codes(c, u[0]);
        }
    }
    if (t == 0) {
        const float r = NORM ? 1.0f / sqrtf(s.ss / (float)cols + a.eps) : 1.0f, y = peak * r;   // the largest value of the normalised row
        a.scale[row] = y < INFINITY ? y / 127.0f : (peak / 127.0f) * r;   // (it may pass fp32 where its 127th part does not)
    }
}

template <class T, bool NORM, int TPR, int PER>
void launch_rows(QrTokenArgs a, hipStream_t st)
{
    constexpr int THREADS = TPR < 128 ? 256 : TPR, RPB = THREADS / TPR;
    constexpr int64_t MOST = ((int64_t)1 << 31) / THREADS * RPB;   // rows of a launch: a grid has less than 2^32 threads
    for (int64_t left = a.rows; left > 0; left -= MOST) {
        a.rows = left < MOST ? left : MOST;
        tokens_kernel<T, NORM, TPR, PER><<<(unsigned)((a.rows + RPB - 1) / RPB), THREADS, 0, st>>>(a);
        a.x = (const T *)a.x + MOST * a.ld_x;
        if (a.residual) {
            a.residual = (const T *)a.residual + MOST * a.ld_res;
            a.sum = (T *)a.sum + MOST * a.ld_sum;
        }
        a.q += MOST * a.ld_q;
        a.scale += MOST;
    }
}

template <class T, bool NORM>
void launch_tokens(const QrTokenArgs &a, hipStream_t st)
{
    constexpr int V = QrVec<T>::N;
    // A row to as few threads as its registers allow, and vectors as even as can be: what a wave has beyond the row it skips, but a
    // thread's part of it it computes (us at 4 to 16 thousand rows; a copy of as many bytes): 4096 bf16 with residual 83 (90), 1280 fp32
    // 19.7 by 64 x 5, 20.4 by 128 x 3 (19.7), 2300 bf16 with residual 74 by 64 x 5, 70 by 128 x 3 (51), 2000 fp16 with residual 14.8 by
    // 128 x 2, 17.7 by 256 (10.8), 4104 bf16 with residual 100 by 256 x 3, 113 by 512 x 2 (91), 8192 bf16 with residual 34.9 by 512,
    // 37.2 by 256 (33.1), 12000 bf16 with residual 128 by 512 x 3, 165 by 1024 x 2 (132).
    // Rows of few vectors share a wave: 500000 x 128 bf16 with residual 92 by 16, 344 by 64 (86); 16384 x 256 11.2 by 32, 17.3 by 64.
    const int nv = (a.cols + V - 1) / V;
#define QR_TOKENS(tpr, per) launch_rows<T, NORM, tpr, per>(a, st)
    if constexpr (!NORM && V == 4) {
        if (nv > 256 && nv <= 320) {
            QR_TOKENS(64, 5);
            return;
        }
    }
    if (nv <= 16) QR_TOKENS(16, 1);
    else if (nv <= 32) QR_TOKENS(32, 1);
    else if (nv <= 64) QR_TOKENS(64, 1);
    else if (nv <= 128) QR_TOKENS(64, 2);
    else if (nv <= 256) QR_TOKENS(128, 2);
    else if (nv <= 384) QR_TOKENS(128, 3);
    else if (nv <= 512) QR_TOKENS(256, 2);
    else if (nv <= 768) QR_TOKENS(256, 3);
    else if (nv <= 1024) QR_TOKENS(512, 2);
    else if (nv <= 1536) QR_TOKENS(512, 3);
    else if (nv <= 2048) QR_TOKENS(1024, 2);
    else if (nv <= 4096) QR_TOKENS(1024, 4);
    else QR_TOKENS(1024, 0);
#undef QR_TOKENS
}

template <bool NORM>
qrnnt_status launch_tokens(int dtype, const QrTokenArgs &a, hipStream_t st)
{
    if (dtype == QRNNT_F32) launch_tokens<float, NORM>(a, st);
    else if (dtype == QRNNT_F16) launch_tokens<_Float16, NORM>(a, st);
    else launch_tokens<__bf16, NORM>(a, st);
    return qr_launch_status();
}

}  // namespace

extern "C" qrnnt_status qrnnt_quantize_tokens(const void *x, int32_t dtype, int64_t rows, int32_t cols, int64_t ld_x, int8_t *q,
                                              int32_t ld_q, float *scale, void *stream)
{
    QR_REQUIRE(qr_is_dtype(dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(rows >= 0 && cols > 0 && ld_x >= cols && ld_q >= cols && ld_q % 16 == 0, QRNNT_ERR_SHAPE);
    QR_REQUIRE(qr_counts_ok(rows, cols) && qr_pitch_ok(rows, ld_x), QRNNT_ERR_UNSUPPORTED);
    if (rows == 0) return QRNNT_OK;
    QR_REQUIRE(x != nullptr && q != nullptr && scale != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(qr_aligned(x, qr_dtype_size(dtype)) && qr_aligned(q, 16) && qr_aligned(scale, 4), QRNNT_ERR_ALIGN);
    QrTokenArgs a = {};
    a.x = x;  a.rows = rows;  a.cols = cols;  a.ld_x = ld_x;  a.q = q;  a.ld_q = ld_q;  a.scale = scale;
    return launch_tokens<false>(dtype, a, (hipStream_t)stream);
}

extern "C" qrnnt_status qrnnt_rms_norm_quant(const void *x, const void *residual, const void *weight, int32_t dtype, int64_t rows,
                                             int32_t cols, int64_t ld_x, int64_t ld_residual, float eps, void *sum_out,
                                             int64_t ld_sum, int8_t *q, int32_t ld_q, float *scale, void *stream)
{
    QR_REQUIRE(qr_is_dtype(dtype) && eps >= 0.0f && eps < INFINITY, QRNNT_ERR_RANGE);
    QR_REQUIRE(rows >= 0 && cols > 0 && ld_x >= cols && ld_q >= cols && ld_q % 16 == 0, QRNNT_ERR_SHAPE);
    QR_REQUIRE(residual == nullptr || (ld_residual >= cols && ld_sum >= cols), QRNNT_ERR_SHAPE);
    QR_REQUIRE(qr_counts_ok(rows, cols) && qr_pitch_ok(rows, ld_x), QRNNT_ERR_UNSUPPORTED);
    QR_REQUIRE(residual == nullptr || (qr_pitch_ok(rows, ld_residual) && qr_pitch_ok(rows, ld_sum)), QRNNT_ERR_UNSUPPORTED);
    if (rows == 0) return QRNNT_OK;
    QR_REQUIRE(x != nullptr && q != nullptr && scale != nullptr && (residual == nullptr || sum_out != nullptr), QRNNT_ERR_NULL);
    const size_t e = qr_dtype_size(dtype);
    QR_REQUIRE(qr_aligned(x, e) && qr_aligned(residual, e) && qr_aligned(weight, e) && qr_aligned(sum_out, e) && qr_aligned(q, 16) && qr_aligned(scale, 4),
               QRNNT_ERR_ALIGN);
    if (residual != nullptr) {
        const auto apart = [&](const void *in, int64_t ld) {
            return (sum_out == in && (ld_sum == ld || rows == 1)) || !qr_rows_overlap(sum_out, qr_matrix_bytes(rows, cols, ld_sum, e), cols * e, ld_sum * e,
                                                                       in, qr_matrix_bytes(rows, cols, ld, e), cols * e, ld * e);
        };
        QR_REQUIRE(apart(x, ld_x) && apart(residual, ld_residual), QRNNT_ERR_RANGE);
    }
    QrTokenArgs a = {};
    a.x = x;  a.residual = residual;  a.weight = weight;  a.sum = sum_out;  a.rows = rows;  a.cols = cols;
    a.ld_x = ld_x;  a.ld_res = ld_residual;  a.ld_sum = ld_sum;  a.eps = eps;  a.q = q;  a.ld_q = ld_q;  a.scale = scale;
    return launch_tokens<true>(dtype, a, (hipStream_t)stream);
}
