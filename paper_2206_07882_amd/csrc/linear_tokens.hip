// 8-bit linear layers whose activations have a scale for each row: y[m,r] = a_scale[m] * row_scale[r] * sum + bias[r]
// with exact int32 sums on the matrix units.
#include <atomic>
#include <type_traits>

#include "elem.h"
#include "kernels.h"
#include "mma_pipe.h"

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
    void *part;                   // [parts][M][ld_part] v4i: sums of the parts of a product that is cut along its columns
    int ld_part;
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

// Few tokens: the weights are what is read.  A workgroup has RT tiles of 16 rows x 16*NT tokens; its waves take the 128-column
// chunks in turn (each weight fragment is fetched once, straight into registers) and join their sums through LDS, where wave i
// finishes the row tiles i, i + WAVES, ...
// Grid: x = blocks of 16*RT rows.  Bound by the weights' way from memory: 16 x 32000 x 1024 fp32, 35 MB, 7.4 us (4.7 TB/s with the launch).
template <class T, int RT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_tokens_few_kernel(const QrTokensLinear p)
{
    __shared__ v4i part[WAVES][RT][NT][64];   // [wave that summed][row tile][token tile]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int n_row_tiles = (p.rows + 15) >> 4, rt0 = blockIdx.x * RT;
    const v4i *w[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int rt = rt0 + i < n_row_tiles ? rt0 + i : n_row_tiles - 1;
        w[i] = p.w + (size_t)rt * p.nkc * 128 + lane;
    }
    const int8_t *a[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int m = nt * 16 + col;
        a[nt] = p.a + (int64_t)(m < p.M ? m : p.M - 1) * p.ld_a;
    }
    v4i acc[RT][NT] = {};
#pragma unroll 2
    for (int kc = wave; kc < p.nkc; kc += WAVES) {
        // columns behind the row's pitch: any of its bytes do, they meet the zero padding of the weights
        int k0 = kc * QRNNT_KCHUNK + grp * 16, k1 = k0 + 64;
        k0 = k0 < p.K ? k0 : 0;
        k1 = k1 < p.K ? k1 : 0;
        v4i wf[2][RT], af[2][NT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            wf[0][i] = w[i][(size_t)kc * 128];
            wf[1][i] = w[i][(size_t)kc * 128 + 64];
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            af[0][nt] = *(const v4i *)(a[nt] + k0);
            af[1][nt] = *(const v4i *)(a[nt] + k1);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[i][nt] = qr_mfma(wf[h][i], af[h][nt], acc[i][nt]);
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
        v4i sum = part[0][i][nt][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += part[v][i][nt][lane];
        float sw[4], bs[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = r0 + j < p.rows ? r0 + j : p.rows - 1;
            sw[j] = p.s_w[r];
            bs[j] = p.bias ? p.bias[r] : 0.0f;
        }
        finish<T>(p, m, r0, sum, sw, bs, p.s_a[m]);
    }
}

// One float a lane straight to LDS.
__device__ __forceinline__ void qr_load_lds4(const void *gptr, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(gptr), "s"(lds_addr) : "memory");
}

// Past the caches.  In asm: the compiler makes one ordinary store of a nontemporal and an ordinary one in two branches.
// (s_nop 1: two wait states before the data registers of a wide store may be rewritten.)
__device__ __forceinline__ void store_past(float *p, v4f v)
{
    asm volatile("global_store_dwordx4 %0, %1, off nt\n\ts_nop 1" ::"v"(p), "v"(v) : "memory");
}

// Many tokens: the matrix units are what is kept busy.  A workgroup of WN x WM waves has BN = 16*MT*WN weight rows x
// BM = 16*NT*WM tokens.  LDS holds the weights of 2D steps of 64 columns (1 KiB blocks as the blob has them: operand order) and
// the activations of D chunks of 128 (1 KiB blocks of 8 tokens x 128 bytes, lane l of the loading wave fetching token l/8's
// 16-byte piece (l%8) ^ (l/8): whole lines per load, operand reads spread over the banks).  Both arrive by direct loads to LDS up
// to three steps ahead, and a wave reads the next step's first operands before its last matrix instructions of the present one.
// Bound, large tiles, by the matrix units at the clock that the power leaves them (8192^3 bf16 396 us, 2.78 POP/s: they are busy
// 73 % of the cycles and the clock falls from 2.4 to 1.7 GHz; the library's int8 product of that size reaches 2.06 POP/s) and where
// columns are few by the stores (16384 x 8192 x 128 bf16, 287 MB, 55 us: 5.2 TB/s).  16000 x 2560 x 1280 fp32 takes 65 us: 38
// of products and 31 of stores, half of which pass while the other compute units' tiles are multiplied.
template <int MT, int NT, int WN, int WM, int D>
struct QrTile {
    static constexpr int WAVES = WN * WM, THREADS = 64 * WAVES;
    static constexpr int BN = 16 * MT * WN, BM = 16 * NT * WM;
    static constexpr int A_BLOCKS = MT * WN, B_BLOCKS = 2 * NT * WM;      // of 1 KiB: weights of a step, activations of a chunk
    static constexpr int A_LOADS = A_BLOCKS / WAVES, B_LOADS = B_BLOCKS / WAVES;
    static constexpr int A_STAGE = A_BLOCKS * 1024, B_STAGE = B_BLOCKS * 1024;
    // LDS: the ring, 2 KB for each wave's results, scales and bias of two tiles
    static constexpr int B_AT = 2 * D * A_STAGE, TURN = B_AT + D * B_STAGE, SCALES = TURN + WAVES * 2048;
    static constexpr int SCALE_BYTES = (2 * BN + BM) * 4, LDS = SCALES + 2 * SCALE_BYTES;
    static_assert(A_BLOCKS % WAVES == 0 && B_BLOCKS % WAVES == 0, "every wave loads as much");
    static_assert(D == 2 || D == 4, "ring of chunks");
};

// T: type of y; v4i: the sums themselves go to p.part (a share of a product that is cut along its columns, blockIdx.y).
template <class T, int MT, int NT, int WN, int WM, int D>
__global__ __launch_bounds__(64 * WN * WM) void linear_tokens_kernel(const QrTokensLinear p, int tiles_n, int tiles_m)
{
    using P = QrTile<MT, NT, WN, WM, D>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int wn = wave % WN, wm = wave / WN;
    // Workgroups go to the 8 XCDs in turn; each XCD gets a run of tiles, G blocks of rows side by side, so that what runs on it at a
    // time shares its L2 (G = 2, 4, 8 at 8192^3: 431, 425, 423 us; at 16000 x 2560 x 1280: 78, 79, 84)
    constexpr int G = 4;
    const int total = tiles_n * tiles_m, n_row_tiles = (p.rows + 15) >> 4;
    const unsigned lds0 = (unsigned)(size_t)lds;
    constexpr bool PART = std::is_same<T, v4i>::value;
    const int kc0 = PART ? (int)((int64_t)p.nkc * blockIdx.y / gridDim.y) : 0;
    const int nkc = PART ? (int)((int64_t)p.nkc * (blockIdx.y + 1) / gridDim.y) - kc0 : p.nkc;
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    auto locate = [&](int at, int &rt0, int &m0) {
        const int xcd = at & 7, each = total >> 3, rest = total & 7;
        const int tile = xcd * each + (xcd < rest ? xcd : rest) + (at >> 3);
        const int stripe = tile / (G * tiles_m), in_stripe = tile - stripe * G * tiles_m;
        const int width = tiles_n - stripe * G < G ? tiles_n - stripe * G : G;
        rt0 = (stripe * G + in_stripe % width) * (P::BN / 16);
        m0 = in_stripe / width * P::BM;
    };
    const v4i *src_a[P::A_LOADS];
    const int8_t *src_b[P::B_LOADS];
    auto load_a = [&](int i, int k) {
        const unsigned to = lds0 + (k & (2 * D - 1)) * P::A_STAGE + (wave * P::A_LOADS + i) * 1024;
        qr_load_lds16(src_a[i] + (size_t)k * 64, __builtin_amdgcn_readfirstlane(to));
    };
    auto load_b = [&](int i, int kc) {
        const int c = (kc0 + kc) * QRNNT_KCHUNK;   // columns behind the row: its start instead (they meet zero weights)
        const unsigned to = lds0 + P::B_AT + (kc & (D - 1)) * P::B_STAGE + (wave * P::B_LOADS + i) * 1024;
        qr_load_lds16(src_b[i] + (c + piece < p.K ? c : -piece), __builtin_amdgcn_readfirstlane(to));
    };
    // Order of all loads: A(0), then for every chunk c: B(c), A(2c + 1), A(2c + 2).  Chunks up to D - 2 are on their way before the
    // loop; the two steps of chunk c start B(c + D - 1) and A(2(c + D) - 1), then A(2(c + D)).
    auto load_group = [&](int c) {
#pragma unroll
        for (int i = 0; i < P::B_LOADS; ++i) load_b(i, c);
#pragma unroll
        for (int i = 0; i < P::A_LOADS; ++i) load_a(i, 2 * c + 1);
        if (c + 1 < nkc) {
#pragma unroll
            for (int i = 0; i < P::A_LOADS; ++i) load_a(i, 2 * c + 2);
        }
    };
    // Starts a tile's first loads: its scales and bias (64 to a load, which the waves take in turn), the first chunks.
    auto begin = [&](int rt0, int m0, int scales) {
        if (!PART) {
            constexpr int N_SW = P::BN / 64, N_SA = P::BM / 64;
            for (int j = wave; j < 2 * N_SW + N_SA; j += P::WAVES) {
                const float *src;
                if (j < 2 * N_SW) {
                    const int r = rt0 * 16 + (j % N_SW) * 64 + lane, rr = r < p.rows ? r : p.rows - 1;
                    src = j < N_SW || !p.bias ? p.s_w + rr : p.bias + rr;
                } else {
                    const int m = m0 + (j - 2 * N_SW) * 64 + lane;
                    src = p.s_a + (m < p.M ? m : p.M - 1);
                }
                qr_load_lds4(src, __builtin_amdgcn_readfirstlane(lds0 + scales + j * 256));
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
            src_b[i] = p.a + (int64_t)(m < p.M ? m : p.M - 1) * p.ld_a + piece;
        }
#pragma unroll
        for (int i = 0; i < P::A_LOADS; ++i) load_a(i, 0);
#pragma unroll
        for (int c = 0; c < D - 1; ++c)
            if (c < nkc) load_group(c);
    };
    const char *fa = lds + wn * MT * 1024 + lane * 16;
    const char *fb = lds + P::B_AT + (wm * NT * 2 + (col >> 3)) * 1024 + (col & 7) * 128;
    const int half0 = (grp ^ (col & 7)) * 16, half1 = ((4 + grp) ^ (col & 7)) * 16;

    constexpr int AHEAD = MT > 2 ? 2 : 1;   // weight operands that are read ahead
    v4i acc[MT][NT], b[2][NT] = {}, w[2][MT] = {};
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
    };
    using std::integral_constant;
    // one step of 64 columns.  LA, LB: it starts the loads of weights 2D - 1 steps / activations D - 1 chunks ahead; LEFT: loads that may
    // be in flight when step k + 1 begins (-1: there is none)
    auto step = [&](int k, auto half, auto la, auto lb, auto left) {
        constexpr int h = decltype(half)::value, LEFT = decltype(left)::value;
        constexpr int NB = decltype(lb)::value ? P::B_LOADS : 0, N = NB + (decltype(la)::value ? P::A_LOADS : 0), ROOM = MT - AHEAD;
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
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[i][nt] = qr_mfma(w[h][i], b[h][nt], acc[i][nt]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr integral_constant<int, 0> zero{};
    constexpr integral_constant<int, 1> one{};
    constexpr int A = P::A_LOADS, GROUP = P::B_LOADS + 2 * A;   // loads of a wave: weights of a step, a chunk
    static_assert((D - 1) * GROUP < 64, "the counter of loads has 6 bits");
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
    int scales = P::SCALES;
    begin(rt0, m0, scales);
    // Of several tiles to a workgroup every second compute unit's begin later, by half the time that a tile's stores take: some store
    // while others compute (16384 x 2048 x 1280 fp32 55 us, so 50; 16384 x 4096 x 640 72 and 68; bf16 57 and 54; the tiles of
    // 8192^3 take 100 us each: no difference).
    if (!PART && P::WAVES == 8 && total > (int)gridDim.x && (blockIdx.x >> 3 & 1))
        for (int i = 0; i < 3 * (int)sizeof(T); ++i) __builtin_amdgcn_s_sleep(16);   // (of 1024 cycles)
    for (int at = blockIdx.x;;) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[i][nt] = v4i{};
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
            begin(rt1, m1, 2 * P::SCALES + P::SCALE_BYTES - scales);
        }
        if constexpr (PART) {
            // four rows of a token to a lane: neighbouring lanes' 64 bytes join in the L2, the sums are read again from there
            v4i *part = (v4i *)p.part + (int64_t)blockIdx.y * p.M * p.ld_part;
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
            const float *sc = (const float *)(lds + scales);
            char *turn = lds + P::TURN + wave * 2048;
            constexpr int E = 16 / sizeof(T), MG = 8 / (int)sizeof(T);   // elements of 16 bytes; row tiles whose 128 bytes of a token turn at a time
            typedef T vec_e __attribute__((ext_vector_type(E)));
            typedef T vec_4 __attribute__((ext_vector_type(4)));
            // Rows of whole lines are not kept in the L2 (whose lines the operands are in, and which a launch ends with writing back):
            // large tiles store past it (16384 x 8192 x 512 bf16 95 us, kept or through it 106 and 102), the others through it
            // (1024 x 2048 x 2048 fp32 9.1, past it 9.4, kept 10.1).  Where rows begin inside a line, two stores share it, which
            // only the L2 can join: 11206 x 9400 x 136 bf16 82 us kept, 131 past it; 6000 x 6004 x 200 fp32 44 and 81; 11206 x
            // 9405 x 136 87 and 160.  Small results stay in the caches behind it all the same: 3000 x 1004 x 1000 fp32, 12 MB,
            // 11.1 kept and 10.0 through; 4200 x 4104 x 300 bf16, 34 MB, 17.4 and 19.7.
            const uintptr_t odd = (uintptr_t)p.y | ((uintptr_t)p.ld_y * sizeof(T));
            const bool pieces = (odd & 127) == 0 || ((odd & 15) == 0 && p.M * p.ld_y * (int64_t)sizeof(T) <= 16 << 20);
            v4f sw[MT], bs[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int r = (wn * MT + mt) * 16 + grp * 4;
                sw[mt] = *(const v4f *)(sc + r);
                bs[mt] = p.bias ? *(const v4f *)(sc + P::BN + r) : v4f{};
            }
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
                            else if (MT * WN >= 16) store_past((float *)y, __builtin_bit_cast(v4f, out[i]));
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
                const float sa = sc[2 * P::BN + (wm * NT + nt) * 16 + col];
#pragma unroll
                for (int g = 0; g < MT / MG; ++g) {
#pragma unroll
                    for (int j = 0; j < MG; ++j) {
                        const int mt = g * MG + j;
                        vec_4 v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = (T)fmaf((float)acc[mt][nt][i] * sw[mt][i], sa, bs[mt][i]);
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
        scales = 2 * P::SCALES + P::SCALE_BYTES - scales;
    }
}

// Joins the sums of a product that was cut along its columns: one thread has four rows of a token.
template <class T>
__global__ __launch_bounds__(256) void linear_tokens_join_kernel(const QrTokensLinear p, int n_parts)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)(i / p.ld_part), r0 = (int)(i - (int64_t)m * p.ld_part) * 4;
    if (m >= p.M || r0 >= p.rows) return;
    const v4i *part = (const v4i *)p.part + i;
    v4i sum = *part;
    for (int s = 1; s < n_parts; ++s) sum += part[(int64_t)s * p.M * p.ld_part];
    float sw[4], bs[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = r0 + j < p.rows ? r0 + j : p.rows - 1;
        sw[j] = p.s_w[r];
        bs[j] = p.bias ? p.bias[r] : 0.0f;
    }
    finish<T>(p, m, r0, sum, sw, bs, p.s_a[m]);
}

// How a product is computed: all tokens in one way, or full rounds of large tiles and the tokens that remain in another.
enum QrTokensKind { FEW, SMALL, MIDDLE, LARGE };
struct QrTokensPiece {
    QrTokensKind kind;
    int parts;       // the columns are cut into (SMALL)
    int M;           // tokens
};
struct QrTokensPlan {
    QrTokensPiece piece[2];
    int n;
};

// Tiles by what they were measured to take (us), over 140 layers of 64 to 8192 columns, 64 to 32000 rows and 40 to 16384 tokens (80 % of
// them within a tenth; the kind chosen by it is on average half a per cent slower than the best): a chunk of 128 columns while
// at most half of the places on the device are taken, and with all of them; what a tile costs besides; what a launch does.
// 256 compute units hold one large tile each, or two of the others.
struct QrTileCost {
    int size, places;
    float alone, full, fixed, start;
    float time(int64_t tiles, int chunks) const
    {
        const int64_t rounds = tiles / places, rest = tiles % places;
        return start + rounds * (chunks * full + fixed) + (rest == 0 ? 0.0f : chunks * (rest <= places / 2 ? alone : full) + fixed);
    }
    int64_t tiles(int rows, int M) const { return (int64_t)((rows + size - 1) / size) * ((M + size - 1) / size); }
};
constexpr QrTileCost TILE_COST[] = {{}, {64, 512, 0.26f, 0.43f, 1.1f, 1.9f}, {128, 512, 0.66f, 1.1f, 3.6f, 0.6f}, {256, 256, 1.03f, 1.4f, 9.6f, -1.4f}};

// A sum of few columns is not cut (up to 1920 a launch more costs what eight parts save), nor one whose parts' sums, read and written, pass
// 512 tokens x 128 rows for each chunk of it (the costs above choose 57 thousand at most): so what a call may need is known without its plan.
int most_parts(int nkc) { return nkc < 16 ? 1 : nkc < 32 ? nkc / 4 : 8; }
int64_t most_sums(int nkc) { return (int64_t)nkc << 16; }

// Measured at each choice (us; few / small / middle / large): 32 x 1000 x 1000 (tokens x rows x columns) 3.4 / 4.5; 48 x 16000 x
// 4000 14.1 / 11.9; 200 x 8000 x 500 - / 4.4 / 6.1 / 12.3; 4000 x 1024 x 4096 - / 30.8 / 27.2 / 39.1; 2000 x 5000 x 3000 - / 59 / 46 /
// 37; 8192^3 - / 901 / 584 / 396.  300 x 1024 x 8192 on small tiles whole 21.2, in two parts 15.1, in four 12.9.
QrTokensPiece plan_piece(int rows, int K, int M, float &least)
{
    const int nkc = qr_round_up(K, QRNNT_KCHUNK) / QRNNT_KCHUNK;
    QrTokensPiece best = {SMALL, 1, M};
    least = INFINITY;
    for (int kind = SMALL; kind <= LARGE; ++kind) {
        const QrTileCost &c = TILE_COST[kind];
        for (int parts = 1; parts <= (kind == SMALL ? most_parts(nkc) : 1); ++parts) {
            if (parts > 1 && (int64_t)parts * M * qr_round_up(rows, 4) > most_sums(nkc)) break;
            const float join = parts == 1 ? 0.0f : 3.0f + (float)parts * M * rows * 8 / 4e6f;   // a launch, and the sums written and read at 4 TB/s
            const float t = c.time(c.tiles(rows, M) * parts, (nkc + parts - 1) / parts) + join;
            if (t < least) {
                least = t;
                best = {(QrTokensKind)kind, parts, M};
            }
        }
    }
    return best;
}

// Few tokens: beyond 16 their codes are fetched as often as the weights and more, so long or many rows go to tiles (tokens x rows x
// columns, few / small tiles: 17 x 8192 x 8192 12.4 / 15.1 us; 32 x 32000 x 1024 8.0 / 8.9; 32 x 16384 x 8192 28.8 / 24.9; 48 x 2048 x
// 2048 5.2 / 7.0; 64 x 2048 x 2048 5.8 / 7.0; 64 x 2048 x 4096 9.7 / 8.6)
bool few_tokens(int rows, int K, int M)
{
    return M <= 16 || (M <= 32 && (rows <= 8192 || K <= 2048)) || (M <= 64 && rows <= 4096 && K <= (M <= 48 ? 4096 : 2048));
}

QrTokensPlan plan_linear_tokens(int rows, int K, int M)
{
    if (few_tokens(rows, K, M)) return {{{FEW, 1, M}}, 1};
    float least;
    QrTokensPlan best = {{plan_piece(rows, K, M, least)}, 1};
    // whole rounds of large tiles first, what would leave a round part empty in a launch of its own (6000 x 3000 x 5000: 121 us
    // in two rounds, 96 in one and middle tiles; 2100 x 8192 x 4096 87 and 65)
    const QrTileCost &c = TILE_COST[LARGE];
    const int nkc = qr_round_up(K, QRNNT_KCHUNK) / QRNNT_KCHUNK, across = (rows + c.size - 1) / c.size;
    const int64_t rounds = c.tiles(rows, M) / c.places;
    for (int64_t r = rounds > 1 ? rounds - 1 : rounds; r >= 1 && r <= rounds; ++r) {
        const int64_t first = r * c.places / across * c.size;   // tokens of the whole rounds
        if (first < c.size || first >= M) continue;
        float rest;
        const QrTokensPiece second = plan_piece(rows, K, M - (int)first, rest);
        const float t = c.time(c.tiles(rows, (int)first), nkc) + rest + 3.5f;   // (the second launch waits for the first one's last stores)
        if (t < least) {
            least = t;
            best = {{{LARGE, 1, (int)first}, second}, 2};
        }
    }
    return best;
}

template <class T, int MT, int NT, int WN, int WM, int D>
void launch_tiles(const QrTokensLinear &p, int parts, hipStream_t st)
{
    using P = QrTile<MT, NT, WN, WM, D>;
    const int tn = (p.rows + P::BN - 1) / P::BN, tm = (p.M + P::BM - 1) / P::BM;
    const int places = P::WAVES == 8 ? 256 : 512;   // what 256 compute units hold
    static std::atomic<bool> allowed[QR_MAX_DEVICES];   // per device: more than 64 KiB of LDS
    const int d = qr_current_device();
    if (!allowed[d].load(std::memory_order_relaxed) &&
        hipFuncSetAttribute((const void *)linear_tokens_kernel<T, MT, NT, WN, WM, D>, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS) == hipSuccess)
        allowed[d].store(true, std::memory_order_relaxed);   // (where it failed the launch says so, and the next call asks again)
    linear_tokens_kernel<T, MT, NT, WN, WM, D><<<dim3((unsigned)(tn * tm < places ? tn * tm : places), parts), P::THREADS, P::LDS, st>>>(p, tn, tm);
}

template <class T, int RT, int NT, int WAVES>
void launch_few(const QrTokensLinear &p, hipStream_t st)
{
    linear_tokens_few_kernel<T, RT, NT, WAVES><<<(unsigned)((p.rows + 16 * RT - 1) / (16 * RT)), 64 * WAVES, 0, st>>>(p);
}

template <class T>
void launch_piece(const QrTokensLinear &p, const QrTokensPiece &piece, hipStream_t st)
{
    switch (piece.kind) {
    case FEW:
        // One row tile to a workgroup while that does not take more than about three workgroups a compute unit; 8 waves where there are
        // few of them (1 x 512 x 8192 3.7 us, with 4 waves 4.4; 16 x 8192 x 4096 7.3, with 4 waves 6.8).  Two row tiles beyond (16 x
        // 16384 x 8192 24.3 us, one tile 29.5; 1 x 12000 x 4096 8.9, one tile 8.6).
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
            launch_tiles<v4i, 4, 1, 1, 4, 4>(p, piece.parts, st);
            linear_tokens_join_kernel<T><<<(unsigned)(((int64_t)p.M * p.ld_part + 255) / 256), 256, 0, st>>>(p, piece.parts);
        } else {
            launch_tiles<T, 4, 1, 1, 4, 4>(p, 1, st);
        }
        return;
    case MIDDLE: launch_tiles<T, 4, 4, 2, 2, 2>(p, 1, st); return;
    case LARGE: launch_tiles<T, 8, 4, 2, 4, 2>(p, 1, st); return;
    }
}

template <class T>
void launch_linear_tokens(QrTokensLinear p, const QrTokensPlan &plan, hipStream_t st)
{
    for (int i = 0; i < plan.n; ++i) {
        p.M = plan.piece[i].M;
        launch_piece<T>(p, plan.piece[i], st);
        p.a += (int64_t)p.M * p.ld_a;
        p.s_a += p.M;
        p.y = (T *)p.y + p.M * p.ld_y;
    }
}

bool tokens_weights_ok(const qrnnt_qmat *w) { return w != nullptr && w->rows > 0 && w->rows <= 1 << 28 && w->cols > 0 && w->cols <= 131071; }

}  // namespace

extern "C" size_t qrnnt_linear_tokens_workspace(const qrnnt_qmat *w, int32_t M)
{
    if (!tokens_weights_ok(w) || M <= 0 || M > 1 << 28) return 0;
    // what the largest call of up to M tokens takes: fewer tokens may be cut where these are not
    const int nkc = qr_round_up(w->cols, QRNNT_KCHUNK) / QRNNT_KCHUNK, parts = most_parts(nkc);
    if (parts == 1 || few_tokens(w->rows, w->cols, M)) return 0;
    const int64_t sums = (int64_t)parts * M * qr_round_up(w->rows, 4);
    return (size_t)(sums < most_sums(nkc) ? sums : most_sums(nkc)) * 4;
}

extern "C" qrnnt_status qrnnt_linear_tokens(const qrnnt_qmat *w, const float *bias, const int8_t *a, int32_t ld_a,
                                            const float *a_scale, int32_t M, void *y, int32_t y_dtype, int64_t ld_y,
                                            void *workspace, size_t workspace_bytes, void *stream)
{
    qrnnt_status s = qr_check_qmat(w, QRNNT_LAYOUT_TILED);
    if (s != QRNNT_OK) return s;
    QR_REQUIRE(qr_is_dtype(y_dtype), QRNNT_ERR_RANGE);
    QR_REQUIRE(M >= 0 && ld_a >= qr_act_pitch(w->cols) && ld_a % 16 == 0 && ld_y >= w->rows, QRNNT_ERR_SHAPE);
    QR_REQUIRE(qr_bits(w) == 8 && tokens_weights_ok(w) && M <= 1 << 28 && qr_pitch_ok(M, ld_y), QRNNT_ERR_UNSUPPORTED);
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
    p.part = workspace;  p.ld_part = qr_round_up(w->rows, 4) / 4;
    const QrTokensPlan plan = plan_linear_tokens(w->rows, w->cols, M);
    QR_REQUIRE(plan.piece[0].kind == FEW || TILE_COST[plan.piece[0].kind].tiles(w->rows, M) < 1 << 23, QRNNT_ERR_UNSUPPORTED);   // (a grid has less than 2^32 threads)
    if (y_dtype == QRNNT_F32) launch_linear_tokens<float>(p, plan, (hipStream_t)stream);
    else if (y_dtype == QRNNT_F16) launch_linear_tokens<_Float16>(p, plan, (hipStream_t)stream);
    else launch_linear_tokens<__bf16>(p, plan, (hipStream_t)stream);
    return qr_launch_status();
}
