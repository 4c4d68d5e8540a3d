// Reordering of hypotheses' states after a selection (Sec. 2: a beam's next hypotheses continue from their parents'
// states): row gathers of several arrays in one launch, in place or into a second set of arrays.
#include "elem.h"
#include "kernels.h"

namespace {

struct QrReorderArgs {
    struct {
        const char *src;
        char *dst;
        int64_t row_bytes, src_pitch, dst_pitch;
    } s[QRNNT_MAX_STATES];
    unsigned end[QRNNT_MAX_STATES];   // workgroups up to the end of each array's
    const int32_t *parent;
    int B, W, W_out, n;
};

typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned u32_any __attribute__((aligned(1)));

// A thread owns one piece of PIECE bytes (of the row's last, shorter piece: one byte each) in NR rows of an utterance: it
// reads the pieces of all their parents, then writes them.  With NR >= W_out no other thread touches them, so a row may
// be overwritten in place.
// Bound by memory: 1024 hypotheses with a row in each of 8 arrays, 28 KB together, 57.7 MB read and written, in 8.6 to 10 us (they fit
// the last cache); one beam of 16 takes 4 us, a launch and two dependent loads.  Four rows to a thread: a parent's pieces that
// several children take come from the L1.
template <class PIECE, int NR, bool IN_PLACE>
__global__ __launch_bounds__(256) void reorder_kernel(const QrReorderArgs a)
{
    constexpr int SIZE = sizeof(PIECE);
    int k = 0;
    while (blockIdx.x >= a.end[k]) ++k;   // uniform
    const unsigned block = blockIdx.x - (k ? a.end[k - 1] : 0u);
    const char *src = a.s[k].src;
    char *dst = a.s[k].dst;
    const int64_t whole = a.s[k].row_bytes / SIZE, pieces = whole + a.s[k].row_bytes % SIZE;
    const int groups = IN_PLACE ? 1 : (a.W_out + NR - 1) / NR;
    const int64_t i = (int64_t)block * 256 + threadIdx.x;
    // (quotients of 64 bits take longer than all else here)
    const int64_t bg = i < 1ll << 31 && pieces < 1ll << 31 ? (int64_t)((unsigned)i / (unsigned)pieces) : i / pieces, piece = i - bg * pieces;
    if (bg >= (int64_t)a.B * groups) return;
    const int b = IN_PLACE ? (int)bg : (int)((unsigned)bg / (unsigned)groups), j0 = IN_PLACE ? 0 : ((int)bg - b * groups) * NR;
    const bool single = piece >= whole;   // a byte behind the last whole piece
    const int64_t at = single ? whole * SIZE + (piece - whole) : piece * SIZE;
    const int32_t *parent = a.parent + (int64_t)b * a.W_out + j0;
    const int n = a.W_out - j0 < NR ? a.W_out - j0 : NR;
    int from[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        const int p = j < n ? parent[j] : -1;
        from[j] = p >= a.W ? a.W - 1 : p;
        if (IN_PLACE && p == j) from[j] = -1;   // stays
    }
    const char *s = src + (int64_t)b * a.W * a.s[k].src_pitch + at;
    char *d = dst + ((int64_t)b * a.W_out + j0) * a.s[k].dst_pitch + at;
    if (single) {
        char v[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (from[j] >= 0) v[j] = s[from[j] * a.s[k].src_pitch];
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (from[j] >= 0) d[j * a.s[k].dst_pitch] = v[j];
        return;
    }
    PIECE v[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j)
        if (from[j] >= 0) v[j] = *(const PIECE *)(s + from[j] * a.s[k].src_pitch);
#pragma unroll
    for (int j = 0; j < NR; ++j)
        if (from[j] >= 0) *(PIECE *)(d + j * a.s[k].dst_pitch) = v[j];
}

// Workgroups up to the end of each array's; false where a grid does not hold them.
template <class PIECE, int NR, bool IN_PLACE>
bool plan_reorder(QrReorderArgs &a)
{
    int64_t end = 0;
    for (int k = 0; k < a.n; ++k) {
        const int64_t pieces = a.s[k].row_bytes / (int)sizeof(PIECE) + a.s[k].row_bytes % (int)sizeof(PIECE);
        const int64_t groups = IN_PLACE ? 1 : (a.W_out + NR - 1) / NR;
        if (groups * a.B > INT32_MAX || pieces > INT64_MAX / 256 / groups / a.B) return false;
        end += (pieces * groups * a.B + 255) / 256;
        if (end >= 1 << 24) return false;   // (a grid has less than 2^32 threads)
        a.end[k] = (unsigned)end;
    }
    return true;
}

template <class PIECE, int NR, bool IN_PLACE>
void launch_reorder(const QrReorderArgs &a, hipStream_t st)
{
    reorder_kernel<PIECE, NR, IN_PLACE><<<a.end[a.n - 1], 256, 0, st>>>(a);
}

}  // namespace

extern "C" qrnnt_status qrnnt_reorder_states(const qrnnt_state_rows *states, int32_t n_states, const int32_t *parent, int32_t B,
                                             int32_t W, int32_t W_out, void *stream)
{
    QR_REQUIRE(n_states >= 1 && n_states <= QRNNT_MAX_STATES, QRNNT_ERR_RANGE);
    QR_REQUIRE(B >= 0 && W > 0 && W_out > 0, QRNNT_ERR_SHAPE);
    QR_REQUIRE(W <= 64 && W_out <= 64, QRNNT_ERR_UNSUPPORTED);
    QR_REQUIRE(states != nullptr, QRNNT_ERR_NULL);
    const int64_t rows = (int64_t)B * (W > W_out ? W : W_out);
    for (int k = 0; k < n_states; ++k) {
        const qrnnt_state_rows &s = states[k];
        QR_REQUIRE(s.row_bytes > 0 && s.src_pitch >= s.row_bytes && s.dst_pitch >= s.row_bytes, QRNNT_ERR_SHAPE);
        QR_REQUIRE(qr_pitch_ok(rows, s.src_pitch) && qr_pitch_ok(rows, s.dst_pitch), QRNNT_ERR_UNSUPPORTED);
    }
    if (B == 0) return QRNNT_OK;
    QR_REQUIRE(parent != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(qr_aligned(parent, 4), QRNNT_ERR_ALIGN);
    QrReorderArgs out = {}, in = {};
    out.parent = in.parent = parent;
    out.B = in.B = B;  out.W = in.W = W;  out.W_out = in.W_out = W_out;
    const auto src_bytes = [&](int k) { return qr_matrix_bytes((int64_t)B * W, states[k].row_bytes, states[k].src_pitch, 1); };
    const auto dst_bytes = [&](int k) { return qr_matrix_bytes((int64_t)B * W_out, states[k].row_bytes, states[k].dst_pitch, 1); };
    for (int k = 0; k < n_states; ++k) {
        const qrnnt_state_rows &s = states[k];
        QR_REQUIRE(s.src != nullptr && s.dst != nullptr, QRNNT_ERR_NULL);
        const bool in_place = s.src == s.dst && s.src_pitch == s.dst_pitch && W == W_out;
        for (int j = 0; j < n_states; ++j) {
            const qrnnt_state_rows &o = states[j];
            QR_REQUIRE((j == k && in_place) || !qr_rows_overlap(s.dst, dst_bytes(k), s.row_bytes, s.dst_pitch, o.src, src_bytes(j), o.row_bytes, o.src_pitch),
                       QRNNT_ERR_RANGE);
            QR_REQUIRE(j == k || !qr_rows_overlap(s.dst, dst_bytes(k), s.row_bytes, s.dst_pitch, o.dst, dst_bytes(j), o.row_bytes, o.dst_pitch),
                       QRNNT_ERR_RANGE);
        }
        QR_REQUIRE(!qr_overlap(s.dst, dst_bytes(k), parent, (size_t)B * W_out * 4), QRNNT_ERR_RANGE);
        QrReorderArgs &a = in_place ? in : out;
        a.s[a.n].src = (const char *)s.src;
        a.s[a.n].dst = (char *)s.dst;
        a.s[a.n].row_bytes = s.row_bytes;
        a.s[a.n].src_pitch = s.src_pitch;
        a.s[a.n].dst_pitch = s.dst_pitch;
        ++a.n;
    }
    // in place a thread holds a piece of every row of the beam: of 16 bytes up to 16 rows, of 4 bytes beyond
    const bool narrow = W > 16;
    QR_REQUIRE((plan_reorder<v4u_any, 4, false>(out) && (narrow ? plan_reorder<u32_any, 64, true>(in) : plan_reorder<v4u_any, 16, true>(in))),
               QRNNT_ERR_UNSUPPORTED);
    if (out.n) launch_reorder<v4u_any, 4, false>(out, (hipStream_t)stream);
    if (in.n) narrow ? launch_reorder<u32_any, 64, true>(in, (hipStream_t)stream) : launch_reorder<v4u_any, 16, true>(in, (hipStream_t)stream);
    return qr_launch_status();
}
