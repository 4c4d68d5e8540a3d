// Linear layer of microscaled 4-bit floats: y[m,r] = sum over blocks of 2^(ea + ew) * sum_k a[m,k] w[r,k] + bias[r], on the matrix
// instructions that take both operands' scales (E2M1 codes and E8M0 scales as they are, fp32 sums).
#include <atomic>
#include <type_traits>

#include "elem.h"
#include "mma_pipe.h"
#include "mx4.h"

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

struct QrMx4Linear {
    const v4i *w;                 // codes of the packed weights
    const uint8_t *s_w;           // their scales
    const float *bias;
    int nkc, rows, bytes;         // chunks of 256 columns; bytes of a row of activations that exist
    const uint8_t *a, *s_a;
    int ld_a, ld_sa, M;
    void *y;
    int64_t ld_y;
    void *part;                   // [parts][M][ld_part] v4f: sums of the parts of a product that is cut along its columns
    int ld_part;
};

// D[16 x 16] += A[16 x 128] * B[128 x 16].  Lane l supplies 32 codes of row l%16 of A and column l%16 of B, one block of each, and the
// byte H of sa and sb as their scales; it receives D[4*(l/16) + i][l%16].
template <int H>
__device__ __forceinline__ v4f mfma_mx4(v4i a, v4i b, int sa, int sb, v4f c)
{
    const v8i a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};   // (4-bit operands are the first four registers)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, H, sa, H, sb);
}

// Four neighbouring rows of the layer for one token.
template <class T>
__device__ __forceinline__ void finish(const QrMx4Linear &p, int m, int r0, v4f sum)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    T *y = (T *)p.y + (int64_t)m * p.ld_y + r0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += p.bias && r0 + i < p.rows ? p.bias[r0 + i] : 0.0f;
    if (r0 + 4 <= p.rows && ((uintptr_t)y & (sizeof(v4t) - 1)) == 0) {
        *(v4t *)y = v4t{(T)sum[0], (T)sum[1], (T)sum[2], (T)sum[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r0 + i < p.rows) y[i] = (T)sum[i];
    }
}

// Few tokens: the weights are what is read.  A workgroup has RT tiles of 16 rows x 16*NT tokens; its waves take the chunks of 256
// columns in turn (codes and scales of the weights are fetched once, straight into registers) and join their sums through LDS.
// Grid: x = blocks of 16*RT rows.  Bound by the weights' way from memory and the launch: 1 x 32000 x 1024 fp32, 17.7 MB, 3.3 us (5.3
// TB/s), 16 x 32000 x 1024 bf16, 18.6 MB, 4.4 us.
template <class T, int RT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_mx4_few_kernel(const QrMx4Linear p)
{
    __shared__ v4f part[WAVES][RT][NT][64];   // [wave that summed][row tile][token tile]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int n_row_tiles = (p.rows + 15) >> 4, rt0 = blockIdx.x * RT;
    const v4i *w[RT];
    const uint8_t *sw[RT], *a[NT], *sa[NT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int rt = rt0 + i < n_row_tiles ? rt0 + i : n_row_tiles - 1;
        w[i] = p.w + (size_t)rt * p.nkc * 128 + lane;
        sw[i] = p.s_w + (size_t)rt * p.nkc * 128 + col * 8 + grp * 2;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int m = nt * 16 + col < p.M ? nt * 16 + col : p.M - 1;
        a[nt] = p.a + (int64_t)m * p.ld_a;
        sa[nt] = p.s_a + (int64_t)m * p.ld_sa + grp * 2;
    }
    v4f acc[RT][NT] = {};
#pragma unroll 2
    for (int kc = wave; kc < p.nkc; kc += WAVES) {
        // behind the row: its start instead (finite codes meet zero weights)
        int k0 = kc * 128 + grp * 32, k1 = k0 + 16;
        k0 = k0 < p.bytes ? k0 : 0;
        k1 = k1 < p.bytes ? k1 : 0;
        v4i wf[2][RT], af[2][NT];
        int ws[RT], as[NT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            wf[0][i] = w[i][(size_t)kc * 128];
            wf[1][i] = w[i][(size_t)kc * 128 + 64];
            ws[i] = *(const uint16_t *)(sw[i] + (size_t)kc * 128);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            af[0][nt] = *(const v4i *)(a[nt] + k0);
            af[1][nt] = *(const v4i *)(a[nt] + k1);
            as[nt] = *(const uint16_t *)(sa[nt] + kc * 8);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[i][nt] = mfma_mx4<0>(wf[0][i], af[0][nt], ws[i], as[nt], acc[i][nt]);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[i][nt] = mfma_mx4<1>(wf[1][i], af[1][nt], ws[i], as[nt], acc[i][nt]);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) part[wave][i][nt][lane] = acc[i][nt];
    __syncthreads();
    // the RT x NT tiles of the result are dealt to the waves
    for (int u = wave; u < RT * NT; u += WAVES) {
        const int i = u / NT, nt = u % NT;
        const int r0 = (rt0 + i) * 16 + grp * 4, m = nt * 16 + col;
        if (r0 >= p.rows || m >= p.M) continue;
        v4f sum = part[0][i][nt][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += part[v][i][nt][lane];
        finish<T>(p, m, r0, sum);
    }
}

// Many tokens: the matrix units are what is kept busy.  A workgroup of WN x WM waves has BN = 16*MT*WN weight rows x
// BM = 16*NT*WM tokens.  LDS holds the weights of 2D steps of 128 columns (1 KiB blocks as the packed form has them: operand order),
// the activations of D chunks of 256 (1 KiB blocks of 8 tokens x 128 bytes, whole lines per load; token t of 16 has its 16-byte piece q
// at q ^ (4 (t/8) + (t/2)%2): the lanes 0-3, 12-15 and 20-27, whose 256 bytes are read at a time, and the others likewise, find them in
// different banks) and both scales of D chunks.  All arrive by
// direct loads to LDS up to three steps ahead, and a wave reads the next step's first operands before its last matrix instructions of
// the present one.
// Bound, large tiles, by the clock that the power leaves the matrix units: 8192^3 bf16 240 us, 4.6 PFLOP/s, where the instructions
// alone, from registers, reach 7.0 with random operands and 9.7 with zeros (this kernel with zeros: 190 us).  They are busy 57 % of the
// cycles, at 1.85 GHz; operands of a whole step read a step ahead gave no more (256 us), nor wave tiles of 128 x 128 with one
// wave to a SIMD (287).  Many rows and tokens of few columns by the stores (16000 x 2560 x 1280 fp32, 164 MB, 45 us;
// such stores alone take 31): waits that count the last tile's stores in, so that two steps of the next run before these are through,
// gave nothing (47 us; 8192^3 7 % slower).
template <int MT, int NT, int WN, int WM, int D>
struct QrMx4Tile {
    static constexpr int WAVES = WN * WM, THREADS = 64 * WAVES;
    static constexpr int BN = 16 * MT * WN, BM = 16 * NT * WM;
    static constexpr int AHEAD = MT > 4 ? 1 : 2;   // weight operands that are read ahead of their row tile
    static constexpr int A_BLOCKS = MT * WN, B_BLOCKS = 2 * NT * WM;      // of 1 KiB: weights of a step, activations of a chunk
    static constexpr int SQ = NT < 4 ? 1 : 4;   // token tiles whose scales are read at once
    static constexpr int SA_BLOCKS = MT * WN / 2, SB_BLOCKS = NT * WM / 2;   // of 256 bytes: scales of a chunk
    static constexpr int A_LOADS = A_BLOCKS / WAVES, B_LOADS = B_BLOCKS / WAVES, S_LOADS = (SA_BLOCKS + SB_BLOCKS) / WAVES;
    static constexpr int A_STAGE = A_BLOCKS * 1024, B_STAGE = B_BLOCKS * 1024, S_STAGE = (SA_BLOCKS + SB_BLOCKS) * 256;
    // LDS: the rings, 2 KB for each wave's results, bias of two tiles
    static constexpr int B_AT = 2 * D * A_STAGE, S_AT = B_AT + D * B_STAGE, TURN = S_AT + D * S_STAGE, BIAS = TURN + WAVES * 2048;
    static constexpr int BIAS_BYTES = BN * 4, LDS = BIAS + 2 * BIAS_BYTES;
    static_assert(A_BLOCKS % WAVES == 0 && B_BLOCKS % WAVES == 0 && (SA_BLOCKS + SB_BLOCKS) % WAVES == 0, "every wave loads as much");
    static_assert(MT * WN % 2 == 0 && NT * WM % 2 == 0, "scales of two tiles to a load");
    static_assert(MT % 4 == 0 && NT % SQ == 0, "scales of four tiles to a read");
    static_assert(D == 2 || D == 4, "ring of chunks");
    static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
};

// T: type of y; v4f: the sums themselves go to p.part (a share of a product that is cut along its columns, blockIdx.y).
template <class T, int MT, int NT, int WN, int WM, int D>
__global__ __launch_bounds__(64 * WN * WM) void linear_mx4_kernel(const QrMx4Linear p, int tiles_n, int tiles_m)
{
    using P = QrMx4Tile<MT, NT, WN, WM, D>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int wn = wave % WN, wm = wave / WN;
    // Workgroups go to the 8 XCDs in turn; each XCD gets a run of tiles, G blocks of rows side by side, so that what runs on it at a
    // time shares its L2 and writes long pieces of rows (G = 4, 8, 16: 8192^3 240, 240, 241 us; 8192 x 8192 x 2048 75, 73, 77; 16000 x 2560 x
    // 1280 fp32 46.4, 45.2, 45.3; 8192 x 8192 x 256 fp32 60, 51, 48; 4096 x 16384 x 1024 bf16 55, 46, 46; 2048 x 32000 x 1280 bf16 51, 53, 54)
    constexpr int G = 8;
    const int total = tiles_n * tiles_m, n_row_tiles = (p.rows + 15) >> 4;
    const unsigned lds0 = (unsigned)(size_t)lds;
    constexpr bool PART = std::is_same<T, v4f>::value;
    const int kc0 = PART ? (int)((int64_t)p.nkc * blockIdx.y / gridDim.y) : 0;
    const int nkc = PART ? (int)((int64_t)p.nkc * (blockIdx.y + 1) / gridDim.y) - kc0 : p.nkc;
    auto locate = [&](int at, int &rt0, int &m0) {
        const int xcd = at & 7, each = total >> 3, rest = total & 7;
        const int tile = xcd * each + (xcd < rest ? xcd : rest) + (at >> 3);
        const int stripe = tile / (G * tiles_m), in_stripe = tile - stripe * G * tiles_m;
        const int width = tiles_n - stripe * G < G ? tiles_n - stripe * G : G;
        rt0 = (stripe * G + in_stripe % width) * (P::BN / 16);
        m0 = in_stripe / width * P::BM;
    };
    static_assert(P::B_LOADS % 2 == 0, "a wave's blocks begin with tokens 0 to 7 of a tile");
    auto piece = [&](int i) { return ((lane & 7) ^ ((i & 1) * 4 + (lane >> 4 & 1))) * 16; };
    const v4i *src_a[P::A_LOADS];
    const uint8_t *src_b[P::B_LOADS], *src_s[P::S_LOADS];
    auto load_a = [&](int i, int k) {
        const unsigned to = lds0 + (k & (2 * D - 1)) * P::A_STAGE + (wave * P::A_LOADS + i) * 1024;
        qr_load_lds16(src_a[i] + (size_t)k * 64, __builtin_amdgcn_readfirstlane(to));
    };
    auto load_b = [&](int i, int kc) {   // the last loads are those of scales
        if (i < P::B_LOADS) {
            const int c = (kc0 + kc) * 128;   // pieces behind the row: its start instead (finite codes meet zero weights)
            const unsigned to = lds0 + P::B_AT + (kc & (D - 1)) * P::B_STAGE + (wave * P::B_LOADS + i) * 1024;
            qr_load_lds16(src_b[i] + (c + piece(i) < p.bytes ? c : -piece(i)), __builtin_amdgcn_readfirstlane(to));
        } else {
            const int j = i - P::B_LOADS, at = wave * P::S_LOADS + j;
            const unsigned to = lds0 + P::S_AT + (kc & (D - 1)) * P::S_STAGE + at * 256;
            qr_load_lds4(src_s[j] + (size_t)kc * (at < P::SA_BLOCKS ? 128 : 8), __builtin_amdgcn_readfirstlane(to));
        }
    };
    // loads of a wave: weights of a step, the rest of a chunk, all of it
    constexpr int A = P::A_LOADS, B = P::B_LOADS + P::S_LOADS, GROUP = B + 2 * A;
    static_assert((D - 1) * GROUP < 64, "the counter of loads has 6 bits");
    // Order of all loads: A(0), then for every chunk c: B(c), A(2c + 1), A(2c + 2).  Chunks up to D - 2 are on their way before the
    // loop; the two steps of chunk c start B(c + D - 1) and A(2(c + D) - 1), then A(2(c + D)).
    auto load_group = [&](int c) {
#pragma unroll
        for (int i = 0; i < B; ++i) load_b(i, c);
#pragma unroll
        for (int i = 0; i < A; ++i) load_a(i, 2 * c + 1);
        if (c + 1 < nkc) {
#pragma unroll
            for (int i = 0; i < A; ++i) load_a(i, 2 * c + 2);
        }
    };
    // Starts a tile's first loads: its bias (64 to a load, which the waves take in turn), the first chunks.
    auto begin = [&](int rt0, int m0, int bias) {
        if (!PART && p.bias) {
            for (int j = wave; j < P::BN / 64; j += P::WAVES) {
                const int r = rt0 * 16 + j * 64 + lane;
                qr_load_lds4(p.bias + (r < p.rows ? r : p.rows - 1), __builtin_amdgcn_readfirstlane(lds0 + bias + j * 256));
            }
        }
#pragma unroll
        for (int i = 0; i < P::A_LOADS; ++i) {
            const int t = rt0 + wave * P::A_LOADS + i, rt = t < n_row_tiles ? t : n_row_tiles - 1;
            src_a[i] = p.w + ((size_t)rt * p.nkc + kc0) * 128 + lane;
        }
#pragma unroll
        for (int i = 0; i < P::B_LOADS; ++i) {
            const int m = m0 + (wave * P::B_LOADS + i) * 8 + (lane >> 3);
            src_b[i] = p.a + (int64_t)(m < p.M ? m : p.M - 1) * p.ld_a + piece(i);
        }
#pragma unroll
        for (int j = 0; j < P::S_LOADS; ++j) {
            const int at = wave * P::S_LOADS + j;
            // in LDS: [four tiles][half of the chunk's scales][row of a tile][tile], four bytes each, so that a lane reads four tiles' at once
            const bool w = at < P::SA_BLOCKS;
            const int d = (w ? at : at - P::SA_BLOCKS) * 64 + lane, Q = w ? 4 : P::SQ;
            const int tile = d / (32 * Q) * Q + d % Q, r = d / Q % 16, half = d / (16 * Q) % 2 * 4;
            if (w) {
                const int rt = rt0 + tile < n_row_tiles ? rt0 + tile : n_row_tiles - 1;
                src_s[j] = p.s_w + ((size_t)rt * p.nkc + kc0) * 128 + r * 8 + half;
            } else {
                const int m = m0 + tile * 16 + r;
                src_s[j] = p.s_a + (int64_t)(m < p.M ? m : p.M - 1) * p.ld_sa + kc0 * 8 + half;
            }
        }
#pragma unroll
        for (int i = 0; i < A; ++i) load_a(i, 0);
#pragma unroll
        for (int c = 0; c < D - 1; ++c)
            if (c < nkc) load_group(c);
    };
    const char *fa = lds + wn * MT * 1024 + lane * 16;
    const char *fb = lds + P::B_AT + (wm * NT * 2 + (col >> 3)) * 1024 + (col & 7) * 128;
    const int turn_of = (col >> 3) * 4 + (col >> 1 & 1), half0 = ((2 * grp) ^ turn_of) * 16, half1 = ((2 * grp + 1) ^ turn_of) * 16;
    const char *fsa = lds + P::S_AT + (wn * (MT / 4) * 32 + (grp >> 1) * 16 + col) * 16;
    const char *fsb = lds + P::S_AT + P::SA_BLOCKS * 256 + (wm * (NT / P::SQ) * 32 + (grp >> 1) * 16 + col) * (4 * P::SQ);
    const int mine = (grp & 1) * 16;   // a lane's two scales of four

    constexpr int AHEAD = P::AHEAD;
    v4f acc[MT][NT];
    v4i b[2][NT] = {}, w[2][MT] = {};
    int sw[MT], sa[NT];   // scales of the chunk
    v4i sw_next[MT / 4] = {}, sa_next[(NT + 3) / 4] = {};
    static_assert(P::SQ == 4 || NT <= 4, "scales of token tiles in one vector");
    auto wait = [&](auto left) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(left)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    auto first_reads = [&](int k, auto half) {
        constexpr int h = decltype(half)::value;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) b[h][nt] = *(const v4i *)(fb + ((k >> 1) & (D - 1)) * P::B_STAGE + nt * 2048 + (h ? half1 : half0));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) w[h][j] = *(const v4i *)(fa + (k & (2 * D - 1)) * P::A_STAGE + j * 1024);
        if (h == 0) {
            const int at = ((k >> 1) & (D - 1)) * P::S_STAGE;
            if constexpr (P::SQ == 4) {
#pragma unroll
                for (int q = 0; q < NT / 4; ++q) sa_next[q] = *(const v4i *)(fsb + at + q * 512);
            } else {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) sa_next[0][nt] = *(const int *)(fsb + at + nt * 128);
            }
#pragma unroll
            for (int q = 0; q < MT / 4; ++q) sw_next[q] = *(const v4i *)(fsa + at + q * 512);
        }
    };
    using std::integral_constant;
    // one step of 128 columns.  LA, LB: it starts the loads of weights 2D - 1 steps / activations D - 1 chunks ahead; LEFT: loads that may
    // be in flight when step k + 1 begins (-1: there is none)
    auto step = [&](int k, auto half, auto la, auto lb, auto left) {
        constexpr int h = decltype(half)::value, LEFT = decltype(left)::value;
        constexpr int NB = decltype(lb)::value ? B : 0, N = NB + (decltype(la)::value ? A : 0), ROOM = MT - AHEAD;
        if (h == 0) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sa[nt] = (int)((unsigned)sa_next[nt / 4][nt % 4] >> mine);
#pragma unroll
            for (int i = 0; i < MT; ++i) sw[i] = (int)((unsigned)sw_next[i / 4][i % 4] >> mine);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (i + AHEAD < MT) w[h][i + AHEAD] = *(const v4i *)(fa + (k & (2 * D - 1)) * P::A_STAGE + (i + AHEAD) * 1024);
#pragma unroll
            for (int q = i * N / ROOM; i < ROOM && q < (i + 1) * N / ROOM; ++q) {
                if (q < NB) load_b(q, (k >> 1) + D - 1);
                else load_a(q - NB, k + 2 * D - 1);
            }
            if (i == ROOM && LEFT >= 0) {
                wait(integral_constant<int, LEFT >= 0 ? LEFT : 0>{});
                first_reads(k + 1, integral_constant<int, 1 - h>{});
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[i][nt] = mfma_mx4<h>(w[h][i], b[h][nt], sw[i], sa[nt], acc[i][nt]);
        }
    };
    constexpr integral_constant<int, 0> zero{};
    constexpr integral_constant<int, 1> one{};
    int rt0, m0, kc;
    // the last D chunks, t = 0 .. D - 1 (of less than D: the last of these).  The first one's first step starts the last loads.
    auto last = [&](auto tt) {
        constexpr int t = decltype(tt)::value;
        if (nkc < D - t) return;
        step(2 * kc, zero, integral_constant<int, t == 0>{}, integral_constant<int, t == 0>{}, integral_constant<int, (D - 1 - t) * GROUP>{});
        step(2 * kc + 1, one, zero, zero, integral_constant<int, t == D - 1 ? -1 : (D - 2 - t) * GROUP + A>{});
        ++kc;
    };
    locate(blockIdx.x, rt0, m0);
    int bias = P::BIAS;
    begin(rt0, m0, bias);
    // Of several large tiles to a workgroup every second compute unit's begin later, by half the time that a tile's stores take: some store
    // while others compute (16000 x 2560 x 1280 fp32 53 us, so 47; bf16 39 and 37; 8192 x 8192 x 512 bf16 35 and 32).
    if (!PART && P::WAVES == 8 && total > (int)gridDim.x && (blockIdx.x >> 3 & 1))
        for (int i = 0; i < 3 * (int)sizeof(T); ++i) __builtin_amdgcn_s_sleep(16);   // (of 1024 cycles)
    for (int at = blockIdx.x;;) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[i][nt] = v4f{};
        if (at == (int)blockIdx.x && nkc >= D) wait(integral_constant<int, (D - 2) * GROUP + 2 * A>{});
        else wait(zero);   // (few columns, or the last tile's stores are under way, too)
        first_reads(0, zero);
        for (kc = 0; kc < nkc - D; ++kc) {
            step(2 * kc, zero, one, one, integral_constant<int, (D - 1) * GROUP>{});
            step(2 * kc + 1, one, one, zero, integral_constant<int, (D - 2) * GROUP + 2 * A>{});
        }
        last(zero);
        last(one);
        if constexpr (D == 4) {
            last(integral_constant<int, 2>{});
            last(integral_constant<int, 3>{});
        }
        // the next tile's first loads are under way while this one's results are stored
        at += gridDim.x;
        const bool more = at < total;
        int rt1 = 0, m1 = 0;
        if (more) {
            locate(at, rt1, m1);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();   // all waves have read the ring
            __builtin_amdgcn_sched_barrier(0);
            begin(rt1, m1, 2 * P::BIAS + P::BIAS_BYTES - bias);
        }
        if constexpr (PART) {
            // four rows of a token to a lane: neighbouring lanes' 64 bytes join in the L2, the sums are read again from there
            v4f *part = (v4f *)p.part + (int64_t)blockIdx.y * p.M * p.ld_part;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int m = m0 + (wm * NT + nt) * 16 + col;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const int r4 = (rt0 + wn * MT + mt) * 4 + grp;
                    if (m < p.M && r4 < p.ld_part) part[(int64_t)m * p.ld_part + r4] = acc[mt][nt];
                }
            }
        } else {
            char *turn = lds + P::TURN + wave * 2048;
            constexpr int E = 16 / sizeof(T), MG = 8 / (int)sizeof(T);   // elements of 16 bytes; row tiles whose 128 bytes of a token turn at a time
            typedef T vec_e __attribute__((ext_vector_type(E)));
            typedef T vec_4 __attribute__((ext_vector_type(4)));
            // Rows of whole lines are not kept in the L2 (whose lines the operands are in, and which a launch ends with writing back):
            // large tiles store past it and the cache behind it, the others through it.  (Through, large tiles are as fast or slower where
            // results do not fall on those of the last call: us, past and through, 16000 x 2560 x 1280 fp32 44 / 51, 2048 x 32000 x 2048 fp32
            // 85 / 92, 8192 x 8192 x 1280 bf16 53 / 54.  Into one buffer again and again, which the cache holds, it would be 46 / 44.)  Where rows begin inside a
            // line, two stores share it, which only the L2 can join.  Small results stay in the caches behind it all the same.
            const uintptr_t odd = (uintptr_t)p.y | ((uintptr_t)p.ld_y * sizeof(T));
            const bool pieces = (odd & 127) == 0 || ((odd & 15) == 0 && p.M * p.ld_y * (int64_t)sizeof(T) <= 16 << 20);
            v4f bs[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) bs[mt] = p.bias ? *(const v4f *)(lds + bias + ((wn * MT + mt) * 16 + grp * 4) * 4) : v4f{};
            const int t0 = lane >> 3, r0 = (rt0 + wn * MT) * 16 + (lane & 7) * E, tm0 = m0 + wm * NT * 16 + t0;
            T *const y0 = (T *)p.y + (int64_t)tm0 * p.ld_y + r0;
            // a wave turns 128 bytes of 16 tokens at a time, in LDS of its own and without a wait for others: its LDS instructions take
            // effect in their order, so the next pieces are formed and written while the last ones' reads are under way
            vec_e out[2];
            auto store = [&](int nt, int g) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int t = nt * 16 + i * 8, r = g * MG * 16;
                    T *y = y0 + t * p.ld_y + r;
                    if (tm0 + t < p.M) {
                        if (r0 + r + E <= p.rows) {
                            if (!pieces) *(typename QrVec<T>::any *)y = out[i];
                            else if (MT * WN >= 16) qr_store_past((float *)y, __builtin_bit_cast(v4f, out[i]));
                            else qr_store_through((float *)y, __builtin_bit_cast(v4f, out[i]));
                        } else {
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                if (r0 + r + e < p.rows) y[e] = out[i][e];
                        }
                    }
                }
            };
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int g = 0; g < MT / MG; ++g) {
#pragma unroll
                    for (int j = 0; j < MG; ++j) {
                        const int mt = g * MG + j;
                        vec_4 v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = (T)(acc[mt][nt][i] + bs[mt][i]);
                        const int at = (j * 16 + grp * 4) * (int)sizeof(T);
                        *(vec_4 *)(turn + col * 128 + (((at >> 4) ^ (col & 7)) << 4) + (at & 15)) = v;
                    }
                    if (nt + g > 0) store(g > 0 ? nt : nt - 1, g > 0 ? g - 1 : MT / MG - 1);
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int i = 0; i < 2; ++i) out[i] = *(const vec_e *)(turn + (i * 8 + t0) * 128 + (((lane & 7) ^ t0) << 4));
                    __builtin_amdgcn_wave_barrier();
                }
            }
            store(NT - 1, MT / MG - 1);
        }
        if (!more) return;
        rt0 = rt1;
        m0 = m1;
        bias = 2 * P::BIAS + P::BIAS_BYTES - bias;
    }
}

// Joins the sums of a product that was cut along its columns: one thread has four rows of a token.
template <class T>
__global__ __launch_bounds__(256) void linear_mx4_join_kernel(const QrMx4Linear p, int n_parts)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)(i / p.ld_part), r0 = (int)(i - (int64_t)m * p.ld_part) * 4;
    if (m >= p.M || r0 >= p.rows) return;
    const v4f *part = (const v4f *)p.part + i;
    v4f sum = *part;
    for (int s = 1; s < n_parts; ++s) sum += part[(int64_t)s * p.M * p.ld_part];
    finish<T>(p, m, r0, sum);
}

// How a product is computed: all tokens in one way, or full rounds of large tiles and the tokens that remain in another.
enum QrMx4Kind { FEW, SMALL, MIDDLE, LARGE };
struct QrMx4Piece {
    QrMx4Kind kind;
    int parts;       // the columns are cut into (SMALL)
    int M;           // tokens
};
struct QrMx4Plan {
    QrMx4Piece piece[2];
    int n;
};

// What tiles take (us), fitted to 5166 layers of 40 to 8192 columns, 48 to 32000 rows and 17 to 16384 tokens (80 % of the times within 8, 12
// and 15 % of it; the kind and number of parts chosen by it are on average 0.4 % slower than the best): a chunk of 256 columns while
// at most half of the places on the device are taken, and with all of them; what a tile costs besides, and for each byte of a
// result; what a launch does.  256 compute units hold one large tile each, or two of the others.
struct QrTileCost {
    int size, places;
    float alone, full, fixed, byte, start;
    float time(int64_t tiles, int chunks, int bytes) const
    {
        const int64_t rounds = tiles / places, rest = tiles % places, half = places / 2;
        const float each = fixed + byte * bytes, last = alone + (rest > half ? (full - alone) * (rest - half) / half : 0.0f);
        return start + rounds * (chunks * full + each) + (rest == 0 ? 0.0f : chunks * last + each);
    }
    int64_t tiles(int rows, int M) const { return (int64_t)((rows + size - 1) / size) * ((M + size - 1) / size); }
};
constexpr QrTileCost TILE_COST[] = {{}, {64, 512, 0.31f, 0.56f, 0.78f, 0.12f, 2.1f}, {128, 512, 0.70f, 1.40f, 1.0f, 0.53f, 1.7f},
                                    {256, 256, 1.14f, 1.89f, 4.0f, 0.70f, 1.7f}};

// A sum of few columns is not cut, nor one whose parts' sums, read and written, pass 512 tokens x 128 rows for each chunk of it: so
// what a call may need is known without its plan.
int most_parts(int nkc) { return nkc < 16 ? 1 : nkc < 32 ? nkc / 4 : 8; }
int64_t most_sums(int nkc) { return (int64_t)nkc << 16; }

// Measured at each choice (us, bf16; small / middle / large): 1000 x 1000 x 1000 (tokens x rows x columns) 4.4 / 6.8 / 11.7; 128 x 32000 x 1024 7.9 /
// 6.6 / 10.0; 4000 x 1024 x 4096 20 / 15 / 24; 2000 x 5000 x 3000 40 / 28 / 25.  256 x 256 x 8192 on small tiles whole 13.2, in four parts 8.4.
QrMx4Piece plan_piece(int rows, int nkc, int M, int bytes, float &least)
{
    QrMx4Piece best = {SMALL, 1, M};
    least = INFINITY;
    for (int kind = SMALL; kind <= LARGE; ++kind) {
        const QrTileCost &c = TILE_COST[kind];
        for (int parts = 1; parts <= (kind == SMALL ? most_parts(nkc) : 1); ++parts) {
            if (parts > 1 && (int64_t)parts * M * qr_round_up(rows, 4) > most_sums(nkc)) break;
            const float join = parts == 1 ? 0.0f : 1.0f + (float)parts * M * rows * 4e-6f;   // a launch, and the sums written and read
            const float t = c.time(c.tiles(rows, M) * parts, (nkc + parts - 1) / parts, parts == 1 ? bytes : 4) + join;
            if (t < least) {
                least = t;
                best = {(QrMx4Kind)kind, parts, M};
            }
        }
    }
    return best;
}

// Few tokens: beyond 32 their codes are fetched as often as the weights and more, so long or many rows go to tiles.  Few against the best
// tiles, in time: 17 to 32 tokens 0.5 to 0.9 (over 16384 rows and 4096 columns 1.04); 33 to 48 0.6 to 0.9 up to 4096 rows, 0.8 to 8192 (over 4096
// columns 1.1), 0.9 to 16384 of up to 512 columns, 1.05 and more beyond; 49 to 64 0.7 to 0.9 up to 4096 rows, 0.8 to 8192 and 0.9 to 16384 of up to 512
// columns, 1.0 and more beyond.
bool few_tokens(int rows, int K, int M)
{
    if (M <= 32) return true;
    if (M <= 48) return rows <= 4096 || (rows <= 8192 && K <= 4096) || (rows <= 16384 && K <= 512);
    return M <= 64 && (rows <= 4096 || (rows <= 16384 && K <= 512));
}

QrMx4Plan plan_linear(int rows, int K, int M, int bytes)
{
    if (few_tokens(rows, K, M)) return {{{FEW, 1, M}}, 1};
    const int nkc = qr_mx4_chunks(K);
    float least;
    QrMx4Plan best = {{plan_piece(rows, nkc, M, bytes, least)}, 1};
    // whole rounds of large tiles first, what would leave a round part empty in a launch of its own
    const QrTileCost &c = TILE_COST[LARGE];
    const int across = (rows + c.size - 1) / c.size;
    const int64_t rounds = c.tiles(rows, M) / c.places;
    for (int64_t r = rounds > 1 ? rounds - 1 : rounds; r >= 1 && r <= rounds; ++r) {
        const int64_t first = r * c.places / across * c.size;   // tokens of the whole rounds
        if (first < c.size || first >= M) continue;
        float rest;
        const QrMx4Piece second = plan_piece(rows, nkc, M - (int)first, bytes, rest);
        const float t = c.time(c.tiles(rows, (int)first), nkc, bytes) + rest + 2.0f;   // (the second launch waits for the first one's last stores)
        if (t < least) {
            least = t;
            best = {{{LARGE, 1, (int)first}, second}, 2};
        }
    }
    return best;
}

template <class T, int MT, int NT, int WN, int WM, int D>
void launch_tiles(const QrMx4Linear &p, int parts, hipStream_t st)
{
    using P = QrMx4Tile<MT, NT, WN, WM, D>;
    const int tn = (p.rows + P::BN - 1) / P::BN, tm = (p.M + P::BM - 1) / P::BM;
    const int places = P::LDS > 80 * 1024 ? 256 : 512;   // what 256 compute units hold
    static std::atomic<bool> allowed[QR_MAX_DEVICES];   // per device: more than 64 KiB of LDS
    const int d = qr_current_device();
    if (!allowed[d].load(std::memory_order_relaxed) &&
        hipFuncSetAttribute((const void *)linear_mx4_kernel<T, MT, NT, WN, WM, D>, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS) == hipSuccess)
        allowed[d].store(true, std::memory_order_relaxed);   // (where it failed the launch says so, and the next call asks again)
    linear_mx4_kernel<T, MT, NT, WN, WM, D><<<dim3((unsigned)(tn * tm < places ? tn * tm : places), parts), P::THREADS, P::LDS, st>>>(p, tn, tm);
}

template <class T, int RT, int NT, int WAVES>
void launch_few(const QrMx4Linear &p, hipStream_t st)
{
    linear_mx4_few_kernel<T, RT, NT, WAVES><<<(unsigned)((p.rows + 16 * RT - 1) / (16 * RT)), 64 * WAVES, 0, st>>>(p);
}

template <class T>
void launch_piece(const QrMx4Linear &p, const QrMx4Piece &piece, hipStream_t st)
{
    switch (piece.kind) {
    case FEW:
        if (p.M <= 16) {
            if (p.rows <= 4096) launch_few<T, 1, 1, 8>(p, st);
            else if (p.rows <= 12288) launch_few<T, 1, 1, 4>(p, st);
            else launch_few<T, 2, 1, 4>(p, st);
        } else if (p.M <= 32) {
            if (p.rows <= 4096) launch_few<T, 1, 2, 4>(p, st);
            else launch_few<T, 2, 2, 4>(p, st);
        } else {
            launch_few<T, 1, 4, 4>(p, st);
        }
        return;
    case SMALL:
        if (piece.parts > 1) {
            launch_tiles<v4f, 4, 1, 1, 4, 4>(p, piece.parts, st);
            linear_mx4_join_kernel<T><<<(unsigned)(((int64_t)p.M * p.ld_part + 255) / 256), 256, 0, st>>>(p, piece.parts);
        } else {
            launch_tiles<T, 4, 1, 1, 4, 4>(p, 1, st);
        }
        return;
    case MIDDLE: launch_tiles<T, 4, 4, 2, 2, 2>(p, 1, st); return;
    case LARGE: launch_tiles<T, 8, 4, 2, 4, 2>(p, 1, st); return;
    }
}

template <class T>
void launch_linear(QrMx4Linear p, const QrMx4Plan &plan, hipStream_t st)
{
    for (int i = 0; i < plan.n; ++i) {
        p.M = plan.piece[i].M;
        launch_piece<T>(p, plan.piece[i], st);
        p.a += (int64_t)p.M * p.ld_a;
        p.s_a += (int64_t)p.M * p.ld_sa;
        p.y = (T *)p.y + p.M * p.ld_y;
    }
}

bool weights_ok(const qrnnt_mx4 *w) { return w != nullptr && qrnnt_pack_mx4_bytes(w->rows, w->cols) > 0; }

}  // namespace

extern "C" size_t qrnnt_linear_mx4_workspace(const qrnnt_mx4 *w, int32_t M)
{
    if (!weights_ok(w) || M <= 0 || M > 1 << 28) return 0;
    // what the largest call of up to M tokens takes: fewer tokens may be cut where these are not
    const int nkc = qr_mx4_chunks(w->cols), parts = most_parts(nkc);
    if (parts == 1 || few_tokens(w->rows, w->cols, M)) return 0;
    const int64_t sums = (int64_t)parts * M * qr_round_up(w->rows, 4);
    return (size_t)(sums < most_sums(nkc) ? sums : most_sums(nkc)) * 4;
}

extern "C" qrnnt_status qrnnt_linear_mx4(const qrnnt_mx4 *w, const float *bias, const uint8_t *a, int32_t ld_a, const uint8_t *a_scale,
                                         int32_t ld_scale, int32_t M, void *y, int32_t y_dtype, int64_t ld_y, void *workspace,
                                         size_t workspace_bytes, void *stream)
{
    QR_REQUIRE(w != nullptr && w->packed != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(w->rows > 0 && w->cols > 0, QRNNT_ERR_SHAPE);
    QR_REQUIRE(qr_is_dtype(y_dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(weights_ok(w) && M <= 1 << 28 && qr_pitch_ok(M, ld_y), QRNNT_ERR_UNSUPPORTED);
    QR_REQUIRE(M >= 0 && ld_y >= w->rows && ld_a >= qr_mx4_pitch(w->cols) && ld_a % 16 == 0 && ld_scale >= qr_mx4_scale_pitch(w->cols) &&
                   ld_scale % 8 == 0, QRNNT_ERR_SHAPE);
    if (M == 0) return QRNNT_OK;
    QR_REQUIRE(a != nullptr && a_scale != nullptr && y != nullptr, QRNNT_ERR_NULL);
    const size_t need = qrnnt_linear_mx4_workspace(w, M);
    QR_REQUIRE(qr_aligned(w->packed, 16) && qr_aligned(a, 16) && qr_aligned(a_scale, 8) && qr_aligned(y, qr_dtype_size(y_dtype)) &&
                   qr_aligned(bias, 4), QRNNT_ERR_ALIGN);
    QR_REQUIRE(need == 0 || workspace != nullptr, QRNNT_ERR_NULL);
    QR_REQUIRE(need == 0 || qr_aligned(workspace, 256), QRNNT_ERR_ALIGN);
    QR_REQUIRE(workspace_bytes >= need, QRNNT_ERR_WORKSPACE);
    QrMx4Linear p = {};
    p.w = (const v4i *)w->packed;  p.s_w = (const uint8_t *)w->packed + qr_mx4_tiles(w->rows, w->cols) * 2048;  p.bias = bias;
    p.nkc = qr_mx4_chunks(w->cols);  p.rows = w->rows;  p.bytes = qr_mx4_pitch(w->cols);
    p.a = a;  p.s_a = a_scale;  p.ld_a = ld_a;  p.ld_sa = ld_scale;  p.M = M;  p.y = y;  p.ld_y = ld_y;
    p.part = workspace;  p.ld_part = qr_round_up(w->rows, 4) / 4;
    const QrMx4Plan plan = plan_linear(w->rows, w->cols, M, (int)qr_dtype_size(y_dtype));
    // (numbers of tiles, and of tiles of a stripe, stay far from the end of 32 bits)
    QR_REQUIRE(plan.piece[0].kind == FEW || TILE_COST[plan.piece[0].kind].tiles(w->rows, M) < 1 << 23, QRNNT_ERR_UNSUPPORTED);
    if (y_dtype == QRNNT_F32) launch_linear<float>(p, plan, (hipStream_t)stream);
    else if (y_dtype == QRNNT_F16) launch_linear<_Float16>(p, plan, (hipStream_t)stream);
    else launch_linear<__bf16>(p, plan, (hipStream_t)stream);
    return qr_launch_status();
}
