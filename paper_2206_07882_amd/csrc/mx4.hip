// Microscaled 4-bit floats: quantizer of rows, the values that codes stand for, and the layout of weights for the matrix units.
//
// s = 2^(floor(log2 max|x|) - 2) for the block, code = x / s rounded to the nearest of E2M1 (ties to even), at most 6 in magnitude.
// Scales are powers of two: nothing but that one rounding happens, so codes are exact.
#include "elem.h"
#include "mx4.h"
#include "select.h"

namespace {

struct QrMx4Args {
    const void *x;       // quantizer: input; values: output
    uint8_t *q, *scale;
    int64_t rows, ld_x;
    int cols, ld_q, ld_s;
    int units;           // of 8 columns in a row
};

// Eight columns of a row to a lane, four lanes to a block; rows follow one another in the lanes.  (Two, four or eight such places to a
// lane: 16000 x 1280 bf16 11.2, 12.2, 14.5 us, one 10.6.)
struct QrMx4Place {
    int64_t row;
    int col;
    __device__ __forceinline__ explicit QrMx4Place(const QrMx4Args &a)
    {
        const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / a.units;
        const unsigned at = (unsigned)(first - row0 * a.units) + threadIdx.x, r = at / (unsigned)a.units;
        row = row0 + r;
        col = (int)(at - r * (unsigned)a.units) * 8;
    }
};

template <class T>
__device__ __forceinline__ void load8(const T *x, int n, float (&v)[8])
{
    constexpr int V = QrVec<T>::N;
#pragma unroll
    for (int h = 0; h < 8 / V; ++h) {
        float part[V];
        qr_load_vec(x + h * V, n - h * V, 0.0f, part);
#pragma unroll
        for (int i = 0; i < V; ++i) v[h * V + i] = part[i];
    }
}

// A float with the exponent byte of a scale.
__device__ __forceinline__ float scale_value(unsigned e)
{
    return __uint_as_float(e == 0u ? 0x00400000u : e == QR_MX4_NAN ? 0x7FC00000u : e << 23);
}

// Bound by memory: 16000 x 1280 bf16, 52 MB, 10.6 us (4.9 TB/s), 16384 x 8192 bf16, 340 MB, 63 us (5.4 TB/s).
template <class T>
__global__ __launch_bounds__(256) void quantize_mx4_kernel(const QrMx4Args a)
{
    const QrMx4Place p(a);
    float v[8];
    load8((const T *)a.x + p.row * a.ld_x + p.col, p.row < a.rows ? a.cols - p.col : 0, v);
    unsigned key = 0u;   // largest magnitude as bits: NaN above infinity above numbers
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned k = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        key = k > key ? k : key;
    }
    key = qr_quad_max(key);
    // the exponent, less two; below 2^-125 the scale stays at its smallest
    unsigned e = key >> 23;
    const bool finite = e < 255u;
    e = key == 0u ? 127u : !finite ? QR_MX4_NAN : e > 2u ? e - 2u : 0u;
    const float s = scale_value(finite ? e : 127u);
    unsigned c = 0u;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);   // (divides by s, rounds to nearest even, stops at 6)
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    c = finite ? c : 0u;
    // four blocks' scales to the first of 16 lanes
    unsigned four = e;
    four |= (unsigned)__builtin_amdgcn_update_dpp(0, (int)e, 0x104, 0xf, 0xf, true) << 8;    // row_shl:4
    four |= (unsigned)__builtin_amdgcn_update_dpp(0, (int)e, 0x108, 0xf, 0xf, true) << 16;   // row_shl:8
    four |= (unsigned)__builtin_amdgcn_update_dpp(0, (int)e, 0x10C, 0xf, 0xf, true) << 24;   // row_shl:12
    if (p.row >= a.rows) return;
    if (p.col < (a.cols + 31) / 32 * 32) *(unsigned *)(a.q + p.row * a.ld_q + (p.col >> 1)) = c;
    if ((threadIdx.x & 15) == 0) *(unsigned *)(a.scale + p.row * a.ld_s + (p.col >> 5)) = four;
}

// Bound by memory: 16384 x 8192 to bf16, 340 MB, 47 us (7.3 TB/s).
template <class T>
__global__ __launch_bounds__(256) void dequantize_mx4_kernel(const QrMx4Args a)
{
    const QrMx4Place p(a);
    if (p.row >= a.rows) return;
    const unsigned c = *(const unsigned *)(a.q + p.row * a.ld_q + (p.col >> 1));
    const float s = scale_value(a.scale[p.row * a.ld_s + (p.col >> 5)]);
    typedef float v2f __attribute__((ext_vector_type(2)));
    const v2f w[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3)};
    constexpr int V = QrVec<T>::N;
    T *x = (T *)a.x + p.row * a.ld_x + p.col;
#pragma unroll
    for (int h = 0; h < 8 / V; ++h) {
        float part[V];
#pragma unroll
        for (int i = 0; i < V; ++i) part[i] = w[(h * V + i) / 2][(h * V + i) & 1] * s;
        qr_store_vec(x + h * V, a.cols - p.col - h * V, part);
    }
}

struct QrMx4Pack {
    const uint8_t *q, *scale;
    int ld_q, ld_s, rows, cols, blocks, chunks;
    uint8_t *out;
    size_t tiles;
};

// One thread to 16 bytes of codes; the first of every two also to a lane's two scales.  Bound by memory: 8192 x 8192, 71 MB, 15.5 us (4.6 TB/s).
__global__ __launch_bounds__(256) void pack_mx4_kernel(const QrMx4Pack a)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.tiles * 128) return;
    const size_t tile = i >> 7;
    const int lane = i & 63, h = (int)(i >> 6) & 1;
    const int64_t row = (int64_t)(tile / a.chunks) * 16 + (lane & 15);
    const int b = (int)(tile % a.chunks) * 8 + (lane >> 4) * 2;
    v4i c = {};
    if (row < a.rows && b + h < a.blocks) {
        c = *(const v4i *)(a.q + row * a.ld_q + (b + h) * 16);
        const int n = a.cols - (b + h) * QR_MX4_BLOCK;   // columns of the block that exist
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int left = n - d * 8;
            if (left < 8) c[d] = left <= 0 ? 0 : (int)((unsigned)c[d] & ((1u << (4 * left)) - 1u));
        }
    }
    *(v4i *)(a.out + i * 16) = c;
    if (h == 0) {
        unsigned two = 0u;
#pragma unroll
        for (int j = 0; j < 2; ++j) two |= (row < a.rows && b + j < a.blocks ? (unsigned)a.scale[row * a.ld_s + b + j] : 127u) << (8 * j);
        *(uint16_t *)(a.out + a.tiles * 2048 + tile * 128 + (lane & 15) * 8 + (lane >> 4) * 2) = (uint16_t)two;
    }
}

// Launches of at most 2^23 workgroups, by rows (a grid has less than 2^32 threads).
template <class Launch>
void by_rows(QrMx4Args a, size_t size, Launch &&launch)
{
    const int64_t most = ((int64_t)1 << 31) / a.units, rows = a.rows;
    for (int64_t r = 0; r < rows; r += most) {
        a.rows = rows - r < most ? rows - r : most;
        launch(a, (unsigned)((a.rows * a.units + 255) / 256));
        a.x = (const char *)a.x + (size_t)(a.rows * a.ld_x) * size;
        a.q += a.rows * a.ld_q;
        a.scale += a.rows * a.ld_s;
    }
}

qrnnt_status check_mx4(const void *q, int ld_q, const void *scale, int ld_s, int32_t dtype, int64_t rows, int cols, int64_t ld_x)
{
    QR_REQUIRE(qr_is_dtype(dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(rows >= 0 && cols > 0 && ld_x >= cols, QRNNT_ERR_SHAPE);
    QR_REQUIRE(qr_counts_ok(rows, cols) && qr_pitch_ok(rows, ld_x), QRNNT_ERR_UNSUPPORTED);
    QR_REQUIRE(ld_q >= qr_mx4_pitch(cols) && ld_q % 16 == 0 && ld_s >= qr_mx4_scale_pitch(cols) && ld_s % 8 == 0, QRNNT_ERR_SHAPE);
    QR_REQUIRE(rows == 0 || (q != nullptr && scale != nullptr), QRNNT_ERR_NULL);
    QR_REQUIRE(rows == 0 || (qr_aligned(q, 16) && qr_aligned(scale, 8)), QRNNT_ERR_ALIGN);
    return QRNNT_OK;
}

}  // namespace

extern "C" int32_t qrnnt_mx4_pitch(int32_t cols) { return cols > 0 && cols <= 1 << 30 ? qr_mx4_pitch(cols) : 0; }
extern "C" int32_t qrnnt_mx4_scale_pitch(int32_t cols) { return cols > 0 && cols <= 1 << 30 ? qr_mx4_scale_pitch(cols) : 0; }

extern "C" qrnnt_status qrnnt_quantize_mx4(const void *x, int32_t dtype, int64_t rows, int32_t cols, int64_t ld_x, uint8_t *q,
                                           int32_t ld_q, uint8_t *scale, int32_t ld_scale, void *stream)
{
    const qrnnt_status s = check_mx4(q, ld_q, scale, ld_scale, dtype, rows, cols, ld_x);
    if (s != QRNNT_OK || rows == 0) return s;
    QR_REQUIRE(x != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(qr_aligned(x, qr_dtype_size(dtype)), QRNNT_ERR_ALIGN);
    QrMx4Args a = {x, q, scale, rows, ld_x, cols, ld_q, ld_scale, qr_mx4_scale_pitch(cols) * 4};
    by_rows(a, qr_dtype_size(dtype), [&](const QrMx4Args &part, unsigned grid) {
        if (dtype == QRNNT_F32) quantize_mx4_kernel<float><<<grid, 256, 0, (hipStream_t)stream>>>(part);
        else if (dtype == QRNNT_F16) quantize_mx4_kernel<_Float16><<<grid, 256, 0, (hipStream_t)stream>>>(part);
        else quantize_mx4_kernel<__bf16><<<grid, 256, 0, (hipStream_t)stream>>>(part);
    });
    return qr_launch_status();
}

extern "C" qrnnt_status qrnnt_dequantize_mx4(const uint8_t *q, int32_t ld_q, const uint8_t *scale, int32_t ld_scale, int64_t rows,
                                             int32_t cols, void *x, int32_t dtype, int64_t ld_x, void *stream)
{
    const qrnnt_status s = check_mx4(q, ld_q, scale, ld_scale, dtype, rows, cols, ld_x);
    if (s != QRNNT_OK || rows == 0) return s;
    QR_REQUIRE(x != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(qr_aligned(x, qr_dtype_size(dtype)), QRNNT_ERR_ALIGN);
    QrMx4Args a = {x, (uint8_t *)q, (uint8_t *)scale, rows, ld_x, cols, ld_q, ld_scale, (int)(((int64_t)cols + 7) / 8)};
    by_rows(a, qr_dtype_size(dtype), [&](const QrMx4Args &part, unsigned grid) {
        if (dtype == QRNNT_F32) dequantize_mx4_kernel<float><<<grid, 256, 0, (hipStream_t)stream>>>(part);
        else if (dtype == QRNNT_F16) dequantize_mx4_kernel<_Float16><<<grid, 256, 0, (hipStream_t)stream>>>(part);
        else dequantize_mx4_kernel<__bf16><<<grid, 256, 0, (hipStream_t)stream>>>(part);
    });
    return qr_launch_status();
}

extern "C" size_t qrnnt_pack_mx4_bytes(int32_t rows, int32_t cols)
{
    if (rows <= 0 || cols <= 0 || rows > 1 << 28 || cols > QRNNT_MX4_MAX_COLS) return 0;
    return qr_mx4_tiles(rows, cols) <= 1 << 24 ? qr_mx4_packed_bytes(rows, cols) : 0;   // (a grid has less than 2^32 threads)
}

extern "C" qrnnt_status qrnnt_pack_mx4(const uint8_t *q, int32_t ld_q, const uint8_t *scale, int32_t ld_scale, int32_t rows,
                                       int32_t cols, void *packed_out, void *stream)
{
    QR_REQUIRE(q != nullptr && scale != nullptr && packed_out != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(rows > 0 && cols > 0, QRNNT_ERR_SHAPE);
    QR_REQUIRE(qrnnt_pack_mx4_bytes(rows, cols) > 0, QRNNT_ERR_UNSUPPORTED);
    QR_REQUIRE(ld_q >= qr_mx4_pitch(cols) && ld_q % 16 == 0 && ld_scale >= qr_mx4_blocks(cols), QRNNT_ERR_SHAPE);
    QR_REQUIRE(qr_aligned(q, 16) && qr_aligned(packed_out, 16), QRNNT_ERR_ALIGN);
    QrMx4Pack a = {q, scale, ld_q, ld_scale, rows, cols, qr_mx4_blocks(cols), qr_mx4_chunks(cols), (uint8_t *)packed_out, qr_mx4_tiles(rows, cols)};
    pack_mx4_kernel<<<(unsigned)((a.tiles * 128 + 255) / 256), 256, 0, (hipStream_t)stream>>>(a);
    return qr_launch_status();
}
