// 8-bit linear layers whose activations have a scale for each row: y[m,r] = a_scale[m] * row_scale[r] * sum + bias[r]
// with exact int32 sums on the matrix units.
#include "elem.h"
#include "kernels.h"

namespace {

struct QrTokensLinear {
    const v4i *w;                 // TILED, 8-bit
    const float *s_w, *bias;
    int nkc, rows, K;
    const int8_t *a;
    const float *s_a;
    int ld_a, M;
    void *y;
    int64_t ld_y;
};

// Four neighbouring rows of the layer for one token: the only place where sums are rounded (to fp32, and once more to the
// type of y; each of the two scales and the bias costs a rounding of fp32).
template <class T>
__device__ __forceinline__ void finish(const QrTokensLinear &p, int m, int r0, v4i acc, const float (&sw)[4], const float (&bs)[4], float sa)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmaf((float)acc[i] * sw[i], sa, bs[i]);
    T *y = (T *)p.y + (int64_t)m * p.ld_y + r0;
    if (r0 + 4 <= p.rows && ((uintptr_t)y & (sizeof(v4t) - 1)) == 0) {
        *(v4t *)y = v4t{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r0 + i < p.rows) y[i] = (T)v[i];
    }
}

// Few tokens: the weights are what is read.  A workgroup has 64 rows x 16*NT tokens, its waves take the 128-column chunks in
// turn (each weight fragment is fetched once) and join their sums through LDS; wave i finishes row tile i.
// Grid: x = blocks of 64 rows, y = blocks of 16*NT tokens.
template <class T, int NT>
__global__ __launch_bounds__(256) void linear_tokens_few_kernel(const QrTokensLinear p)
{
    __shared__ v4i part[4][4][NT][64];   // [wave that summed][row tile][token tile]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int n_row_tiles = (p.rows + 15) >> 4, rt0 = blockIdx.x * 4, m0 = blockIdx.y * 16 * NT;
    const v4i *w[4];
#pragma unroll
    for (int mt = 0; mt < 4; ++mt) {
        const int rt = rt0 + mt < n_row_tiles ? rt0 + mt : n_row_tiles - 1;
        w[mt] = p.w + (size_t)rt * p.nkc * 128 + lane;
    }
    const int8_t *a[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int m = m0 + nt * 16 + col;
        a[nt] = p.a + (int64_t)(m < p.M ? m : p.M - 1) * p.ld_a;
    }
    v4i acc[4][NT] = {};
    for (int kc = wave; kc < p.nkc; kc += 4) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            // columns behind the row's pitch: any of its bytes do, they meet the zero padding of the weights
            int k = kc * QRNNT_KCHUNK + half * 64 + grp * 16;
            k = k < p.K ? k : 0;
            v4i wf[4], af[NT];
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) wf[mt] = w[mt][(size_t)kc * 128 + half * 64];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) af[nt] = *(const v4i *)(a[nt] + k);
#pragma unroll
            for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = qr_mfma(wf[mt], af[nt], acc[mt][nt]);
        }
    }
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) part[wave][mt][nt][lane] = acc[mt][nt];
    __syncthreads();
    const int r0 = (rt0 + wave) * 16 + grp * 4;
    if (r0 >= p.rows) return;
    float sw[4], bs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + i < p.rows ? r0 + i : p.rows - 1;
        sw[i] = p.s_w[r];
        bs[i] = p.bias ? p.bias[r] : 0.0f;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int m = m0 + nt * 16 + col;
        const v4i sum = part[0][wave][nt][lane] + part[1][wave][nt][lane] + part[2][wave][nt][lane] + part[3][wave][nt][lane];
        if (m < p.M) finish<T>(p, m, r0, sum, sw, bs, p.s_a[m]);
    }
}

template <class T>
void launch_linear_tokens(const QrTokensLinear &p, hipStream_t st)
{
    const unsigned gx = (unsigned)((p.rows + 63) / 64);
    if (p.M <= 16) linear_tokens_few_kernel<T, 1><<<gx, 256, 0, st>>>(p);
    else if (p.M <= 32) linear_tokens_few_kernel<T, 2><<<gx, 256, 0, st>>>(p);
    else linear_tokens_few_kernel<T, 4><<<dim3(gx, (unsigned)((p.M + 63) / 64)), 256, 0, st>>>(p);
}

bool tokens_weights_ok(const qrnnt_qmat *w) { return w != nullptr && w->rows > 0 && w->cols > 0 && w->cols <= 131071; }

}  // namespace

extern "C" size_t qrnnt_linear_tokens_workspace(const qrnnt_qmat *w, int32_t M)
{
    if (!tokens_weights_ok(w) || M <= 0) return 0;
    return 0;
}

extern "C" qrnnt_status qrnnt_linear_tokens(const qrnnt_qmat *w, const float *bias, const int8_t *a, int32_t ld_a,
                                            const float *a_scale, int32_t M, void *y, int32_t y_dtype, int64_t ld_y,
                                            void *workspace, size_t workspace_bytes, void *stream)
{
    qrnnt_status s = qr_check_qmat(w, QRNNT_LAYOUT_TILED);
    if (s != QRNNT_OK) return s;
    QR_REQUIRE(qr_is_dtype(y_dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(M >= 0 && ld_a >= qr_act_pitch(w->cols) && ld_a % 16 == 0 && ld_y >= w->rows, QRNNT_ERR_SHAPE);
    QR_REQUIRE(qr_bits(w) == 8 && tokens_weights_ok(w), QRNNT_ERR_UNSUPPORTED);
    if (M == 0) return QRNNT_OK;
    QR_REQUIRE(a != nullptr && a_scale != nullptr && y != nullptr, QRNNT_ERR_NULL);
    const size_t e = qr_dtype_size(y_dtype), need = qrnnt_linear_tokens_workspace(w, M);
    QR_REQUIRE(qr_aligned(a, 16) && qr_aligned(y, e) && qr_aligned(a_scale, 4) && qr_aligned(bias, 4), QRNNT_ERR_ALIGN);
    QR_REQUIRE(need == 0 || workspace != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(need == 0 || qr_aligned(workspace, 256), QRNNT_ERR_ALIGN);
    QR_REQUIRE(workspace_bytes >= need, QRNNT_ERR_WORKSPACE);
    QrTokensLinear p = {};
    p.w = (const v4i *)w->packed;  p.s_w = w->row_scale;  p.bias = bias;
    p.nkc = qr_round_up(w->cols, QRNNT_KCHUNK) / QRNNT_KCHUNK;  p.rows = w->rows;  p.K = w->cols;
    p.a = a;  p.s_a = a_scale;  p.ld_a = ld_a;  p.M = M;  p.y = y;  p.ld_y = ld_y;
    if (y_dtype == QRNNT_F32) launch_linear_tokens<float>(p, (hipStream_t)stream);
    else if (y_dtype == QRNNT_F16) launch_linear_tokens<_Float16>(p, (hipStream_t)stream);
    else launch_linear_tokens<__bf16>(p, (hipStream_t)stream);
    return qr_launch_status();
}
