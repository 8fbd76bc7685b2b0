// Frozen products with operands in 8 bits: Y = Q(X) Q(W) and dX = Q(dY) Q(W)^T.
//
// Q keeps values of 4 exponent and 3 mantissa bits (largest 448) and one power of two per block, the smallest that brings the
// block's largest magnitude to 448 or below: blocks of 128 x 128 for the weight, of one row's 128 consecutive elements along the
// contraction for the activations.  The scales are powers of two because that is what the matrix units apply by themselves: one
// v_mfma_scale_f32_16x16x128 takes a 128-deep step of 16 x 16 outputs with a scale per row of either operand, so that the sum over
// the blocks stays in the fp32 accumulators and costs no other instruction.  (A scale per 32 elements is what the instruction has;
// the four of a row are the same here.)
//
// The weight is laid out once, in both orientations, each with its contraction consecutive and padded with zeros to a multiple of
// 128: a forward row is an output column.  So both products are one kernel, and k and n may be anything.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "stream_common.h"

namespace mlora {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kQBlock = 128;
static inline int64_t q_blocks(int64_t x) { return (x + kQBlock - 1) / kQBlock; }
static inline int64_t q_words(int64_t x) { return (q_blocks(x) + 3) / 4; }      // words of four consecutive blocks' scales
static inline int64_t q_align(int64_t b) { return (b + 1023) & ~int64_t(1023); }

// Exponent of the scale of a block whose largest finite magnitude has these bits: 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(uint32_t amax) {
    if (amax == 0u) return 0;
    const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, -127);      // denormal magnitudes
}
// v / 2^e: |e| may pass the exponents a float has, so in two exact steps where that matters
__device__ __forceinline__ float scaled_down(float v, int e) { return ldexpf(v, -e); }
__device__ __forceinline__ uint32_t four_bytes(const float (&v)[4], int e) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled_down(v[0], e), scaled_down(v[1], e), w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled_down(v[2], e), scaled_down(v[3], e), w, true);
    return (uint32_t)w;
}
// magnitude as bits; NaN and Inf are left out, for their scale would leave nothing of the others (the element itself becomes NaN at any scale)
__device__ __forceinline__ uint32_t magnitude(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b >= 0x7f800000u ? 0u : b;
}

// ---- activations -----------------------------------------------------------------------------------------------------------
// Q [rows][kp] bytes, kp = K up to a multiple of 128; scales [words][rows_padded]: a word holds the scale bytes (exponent + 127)
// of four consecutive blocks of a row.  A wavefront takes one word (512 columns) of ROWS rows, all on their way at a time; sixteen lanes a block (fp32: 32).
// PAST: the activations do not fit three quarters of the Infinity Cache and are read past it.  A stream: 8192 x 14336 bf16 (352 MB) 59 us (6 TB/s), 72 with a
// row a wavefront, whose scale is four bytes by themselves in a line; fp32 (587 MB) 103 us, 150 with eight columns next to each other a lane; where ROWS = 8
// leaves the chip to few wavefronts, a row each: 1500 x 2048 fp32 5.6 / 9.0 us.
template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}
// A lane takes pieces of sixteen bytes next to its neighbours': eight columns, or in fp32 four of the word's first half and four of its second.
template <typename T, int ROWS, bool PAST>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* X, int64_t rows, int64_t K, int64_t kp, uint8_t* Q, uint32_t* scales, int64_t rows_padded,
                                                         int32_t words) {
    constexpr int E = kEpc<T>, P = 8 / E, LANES = kQBlock / E;      // columns of a piece, pieces of a lane and row, lanes of a block
    const int word = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (word >= words) return;
    const int64_t row0 = (int64_t)blockIdx.x * ROWS, c = (int64_t)word * 512 + lane * E;
    const int count = (int)min((int64_t)ROWS, rows - row0);
    uint4 p[ROWS][P];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int h = 0; h < P; ++h) {
            const int64_t col = c + h * 64 * E;
            const int valid = (int)max((int64_t)0, min((int64_t)E, K - col));
            if (valid > 0) p[r][h] = load16_row<T, PAST>(X + (row0 + min(r, count - 1)) * K + col, valid, K >= E);
            else p[r][h] = zero4();
        }
    uint32_t mine = 0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (r >= count) break;
        uint32_t w = 0;
#pragma unroll
        for (int h = 0; h < P; ++h) {
            const int64_t col = c + h * 64 * E;
            float v[E];
            unpack16<T>(p[r][h], v);
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) m = max(m, magnitude(v[e]));
            m = dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(m))));      // of sixteen lanes
            if constexpr (LANES == 32) {
                const auto both = __builtin_amdgcn_permlane16_swap(m, m, false, false);
                m = max(both[0], both[1]);
            }
            const int e = scale_exponent(m);
            if (col < kp) {
                uint32_t bytes[E / 4];
#pragma unroll
                for (int k = 0; k < E / 4; ++k) {
                    const float four[4] = {v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]};
                    bytes[k] = four_bytes(four, e);
                }
                __builtin_memcpy(__builtin_assume_aligned(Q + (row0 + r) * kp + col, E), bytes, E);
            }
#pragma unroll
            for (int b = 0; b < 64 / LANES; ++b) w |= (uint32_t)(__builtin_amdgcn_readlane(e, b * LANES) + 127) << (8 * (h * (64 / LANES) + b));
        }
        if (lane == r) mine = w;
    }
    if (lane < count) scales[(int64_t)word * rows_padded + row0 + lane] = mine;
}

// ---- weight ----------------------------------------------------------------------------------------------------------------
struct QuantWeight {
    uint8_t* fwd;          // [n][kp]
    uint32_t* fwd_scales;  // [words of k][blocks of n]
    uint8_t* bwd;          // [k][np]
    uint32_t* bwd_scales;  // [words of n][blocks of k]
    int64_t bytes;
};
static QuantWeight quant_weight(int64_t k, int64_t n, void* buf) {
    const int64_t kp = q_blocks(k) * kQBlock, np = q_blocks(n) * kQBlock;
    uint8_t* p = (uint8_t*)buf;
    QuantWeight w;
    int64_t o = 0;
    w.fwd = p; o += q_align(n * kp);
    w.bwd = p + o; o += q_align(k * np);
    w.fwd_scales = (uint32_t*)(p + o); o += q_align(4 * q_words(k) * q_blocks(n));
    w.bwd_scales = (uint32_t*)(p + o); o += q_align(4 * q_words(n) * q_blocks(k));
    w.bytes = o;
    return w;
}

// One work group per 128 x 128 block; blocks past the edge of the scales' last word write a scale only.
template <typename T>
__global__ __launch_bounds__(256) void quant_weight_kernel(const T* W, int64_t k, int64_t n, QuantWeight q) {
    __shared__ uint8_t tile[128][132];      // [contraction of the forward][output], bytes
    __shared__ uint32_t red[4];
    const int64_t kb = blockIdx.y, nb = blockIdx.x, k0 = kb * kQBlock, n0 = nb * kQBlock;
    const int64_t kblocks = (k + kQBlock - 1) / kQBlock, nblocks = (n + kQBlock - 1) / kQBlock;
    const int tid = threadIdx.x, r0 = tid >> 4, c = (tid & 15) * 8;
    float v[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t row = k0 + r0 + 16 * j;
        const int valid = row < k ? (int)max((int64_t)0, min((int64_t)8, n - n0 - c)) : 0;
        if (valid > 0) {
            unpack(load_piece(W + row * n + n0 + c, valid, n >= kPiece), v[j]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[j][e]));
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
    const int e = scale_exponent(m);
    const int64_t np = nblocks * kQBlock, kp = kblocks * kQBlock;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float lo[4] = {v[j][0], v[j][1], v[j][2], v[j][3]}, hi[4] = {v[j][4], v[j][5], v[j][6], v[j][7]};
        const uint32_t a = four_bytes(lo, e), b = four_bytes(hi, e);
        const int r = r0 + 16 * j;
        *reinterpret_cast<uint32_t*>(&tile[r][c]) = a;
        *reinterpret_cast<uint32_t*>(&tile[r][c + 4]) = b;
        if (k0 + r < k) *reinterpret_cast<uint2*>(q.bwd + (k0 + r) * np + n0 + c) = make_uint2(a, b);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int col = r0 + 16 * j;
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int x = 0; x < 8; ++x) w[x >> 2] |= (uint32_t)tile[c + x][col] << (8 * (x & 3));
        if (n0 + col < n) *reinterpret_cast<uint2*>(q.fwd + (n0 + col) * kp + k0 + c) = make_uint2(w[0], w[1]);
    }
    if (tid == 0) {
        reinterpret_cast<uint8_t*>(q.fwd_scales + (kb >> 2) * nblocks + nb)[kb & 3] = (uint8_t)(e + 127);
        reinterpret_cast<uint8_t*>(q.bwd_scales + (nb >> 2) * kblocks + kb)[nb & 3] = (uint8_t)(e + 127);
    }
}

// Eight bytes as bf16 under a block's scale; `scale`'s exponent bits are the scale byte.  Exact, but for elements below 2^-126 (of a block whose largest is
// below 2^-108), which have fewer bits there or none.
__device__ __forceinline__ bf16x8 widened(int lo, int hi, float scale) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One 128-deep step of a 16 x 16 block under the scale bytes of its rows (lowest byte of sx, sy).  The sums inside an 8-bit matrix instruction are not
// fp32 sums: with random operands they are off by up to 2^-13.5 of the magnitudes' sum, 1.5e-5 .. 5e-5 in norm.  That is well below the
// 2^-8 to which a bf16 output is rounded, and not below fp32's.  So fp32 plans widen the bytes to bf16, which holds every 8-bit value
// times its scale, and take four bf16 instructions a step, whose sums are fp32 sums.  (The scales by themselves, on a step's sum, are two instructions a
// sum more: 4096 x 4096 x 4096 in 128 x 128 tiles 171 us instead of 148.)
__device__ __forceinline__ f32x4 q_mma(i32x8 x, i32x8 y, f32x4 c, uint32_t sx, uint32_t sy) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 0, 0, 0, (int)sx, 0, (int)sy);
}

// ---- product ---------------------------------------------------------------------------------------------------------------
// C[M][N] = A[M][K] B[N][K]^T, A and B bytes with rows of kp, a multiple of 128.
struct QGemmArgs {
    const uint8_t* A; const uint32_t* sa; int64_t sa_ld;
    const uint8_t* B; const uint32_t* sb; int64_t sb_ld;
    void* C; int64_t ldc;
    int32_t M, N, steps;
    int64_t kp;
    int32_t tiles_m, tiles_n;
    int32_t xcd_run;      // see tile_of
};

// Direct global -> LDS load of 4 bytes per lane (lane i's land at lds_base + 4 i), as dma16.
__device__ __forceinline__ void dma4(unsigned voff, const void* sbase, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(sbase), "s"(lds_base) : "memory", "m0");
}

// Tile of a work group.  Tiles are numbered down the rows first in bands of 8 row tiles; 32 consecutive numbers (8 x 4 tiles, 12 operand
// panels) go to one XCD (blockIdx % 8) at a time, so that its CUs share the panels in its L2, and all XCDs work on one band.  Fewer
// than 256 tiles are dealt evenly, xcd_run a XCD.  False: no tile.
__device__ __forceinline__ bool tile_of(const QGemmArgs& g, int& tm, int& tn) {
    const int total = g.tiles_m * g.tiles_n, xcd = blockIdx.x % 8, slot = blockIdx.x / 8;
    const int L = g.xcd_run ? xcd * g.xcd_run + slot : ((slot / 32) * 8 + xcd) * 32 + slot % 32;
    if (L >= total || (g.xcd_run && slot >= g.xcd_run)) return false;
    const int band = L / (8 * g.tiles_n), in_band = L - band * 8 * g.tiles_n, rows = min(8, g.tiles_m - band * 8);
    tm = band * 8 + in_band % rows;
    tn = in_band / rows;
    return true;
}

// Large products: 256 x 256 outputs a work group of four wavefronts (2 x 2, one per SIMD), each 128 x 128 = 8 x 8 blocks of 16 x 16: the accumulators
// fill half of the registers, and a step reads 128 KB of LDS for its 2048 cycles of matrix instructions (eight wavefronts of 128 x 64 read 192 KB,
// three quarters of what the LDS can deliver).  A step's 128 bytes of either operand's 256 rows go through LDS (chunk x of row r at x ^ (r & 7):
// 1 KB-linear direct loads, conflict-free reads), two buffers each.  One wavefront per SIMD has nobody to hide its waits, so all of them lie
// behind matrix instructions: the last two row blocks of a step are multiplied behind the barrier that opens the next step, column block by
// column block, and each column block's fragment is replaced by the next step's as soon as it has been used; by the barrier every
// wavefront holds all it still needs of the step, so that the barrier frees the step's buffers.  The sixteen loads a wavefront owes per step
// follow it one per two instructions, and have 32 more to land.  The rows' scales (a word holds four steps') come with every fourth step.
// 8192 x 4096 x 14336 386 - 397 us (2.42 - 2.49 PFLOP/s; averages of two boxes, the least 348), 8192 x 14336 x 4096 349 - 362 (2.66 - 2.76; 314); a library
// product of 8192^3 reaches 2.74.  The matrix units are busy 0.64 and 0.72 of the time, at 1.9 GHz.
constexpr int QTILE = 256 * 128, QSCALES = 1024 + 256;
constexpr int QE_LD = 128 + 8;                                    // epilogue: row of a wavefront's part (elements)
constexpr int QLDS = 4 * 128 * QE_LD * 2 > 4 * QTILE + 2 * QSCALES ? 4 * 128 * QE_LD * 2 : 4 * QTILE + 2 * QSCALES;

__global__ __launch_bounds__(256, 1) void quant_gemm_kernel(QGemmArgs g) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[QLDS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, g4 = lane >> 4;
    int tm, tn;
    if (!tile_of(g, tm, tn)) return;
    const int m0 = tm * 256, n0 = tn * 256;
    f32x4 acc[8][8];
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int b = 0; b < 8; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};

    unsigned oa[8], ob[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {      // rows past the edge repeat the last one: they only feed outputs that are not stored
        const int row = (wave * 8 + c) * 8 + (lane >> 3), ch = (lane & 7) ^ (lane >> 3);
        oa[c] = (unsigned)((int64_t)(min(m0 + row, g.M - 1) - m0) * g.kp + ch * 16);
        ob[c] = (unsigned)((int64_t)(min(n0 + row, g.N - 1) - n0) * g.kp + ch * 16);
    }
    const char* baseA = uniform_ptr(g.A + (int64_t)m0 * g.kp);
    const char* baseB = uniform_ptr(g.B + (int64_t)n0 * g.kp);
    const char* baseSA = uniform_ptr(g.sa + m0);
    const char* baseSB = uniform_ptr(g.sb);
    const unsigned osb = (unsigned)min(n0 / kQBlock + (lane & 1), (g.N - 1) / kQBlock) * 4u;
    const unsigned lds0 = (unsigned)(uintptr_t)lds, ldsw = lds0 + wave * 8192;
    constexpr unsigned kScale0 = 4 * QTILE;
    // load c of the sixteen of step `to`; past the last step the pointers stay, and the last one is loaded again into buffers that nobody reads
    auto issue = [&](int to, int c) {
        const unsigned dst = ldsw + (to & 1) * 2 * QTILE;
        if (c < 8) dma16(oa[c], baseA, dst + c * 1024);
        else       dma16(ob[c - 8], baseB, dst + QTILE + (c - 8) * 1024);
        if (c == 15) {
            const int64_t step = to + 1 < g.steps ? 128 : 0;
            baseA += step;
            baseB += step;
        }
    };
    auto issue_scales = [&](int t) {   // of the steps t .. t + 3, t a multiple of 4 below g.steps
        const unsigned dst = lds0 + kScale0 + ((t >> 2) & 1) * QSCALES;
        if (wave == 0) dma16(lane * 16, baseSA + (int64_t)(t >> 2) * g.sa_ld * 4, dst);
        else if (wave == 1) dma4(osb, baseSB + (int64_t)(t >> 2) * g.sb_ld * 4, dst + 1024);
    };
    i32x8 fa[4], fb[8];
    uint32_t sa[4] = {127u, 127u, 127u, 127u}, sb = 127u, sb_next = 127u;
#pragma unroll
    for (int k = 0; k < 4; ++k) fa[k] = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) fb[k] = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
    const int x0 = (g4 ^ (l16 & 7)) << 4, x1 = ((4 + g4) ^ (l16 & 7)) << 4;
    const int rowA = (wm * 128 + l16) * 128, rowB = (wn * 128 + l16) * 128 + QTILE;
    auto frag = [&](int at) {
        return __builtin_shufflevector(*reinterpret_cast<const i32x4*>(lds + at + x0), *reinterpret_cast<const i32x4*>(lds + at + x1), 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto rfa = [&](int t, int a) {
        fa[a & 3] = frag((t & 1) * 2 * QTILE + rowA + a * 16 * 128);
        sa[a & 3] = lds[kScale0 + ((t >> 2) & 1) * QSCALES + (wm * 128 + a * 16 + l16) * 4 + (t & 3)];
    };
    auto rfb = [&](int t, int b) { fb[b] = frag((t & 1) * 2 * QTILE + rowB + b * 16 * 128); };
    // operands swapped: a lane ends with four consecutive columns of a row
    auto mma = [&](int a, int b) { acc[a][b] = q_mma(fb[b], fa[a & 3], acc[a][b], sb, sa[a & 3]); };
#define Q_FENCE __builtin_amdgcn_sched_barrier(0)
    issue_scales(0);
#pragma unroll
    for (int c = 0; c < 16; ++c) issue(0, c);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    for (int t = 0; t < g.steps; ++t) {
        if ((t & 3) == 0 && t + 4 < g.steps) issue_scales(t + 4);
        sb_next = lds[kScale0 + ((t >> 2) & 1) * QSCALES + 1024 + wn * 4 + (t & 3)];
        Q_FENCE;
        // the last two row blocks of the step before (zeros at first)
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            issue(t + 1, b);
            Q_FENCE;
            mma(6, b);
            mma(7, b);
            rfb(t, b);
            if (b < 2) rfa(t, b);
            Q_FENCE;
        }
        sb = sb_next;
#pragma unroll
        for (int a = 0; a < 6; ++a) {
            rfa(t, a + 2);
            Q_FENCE;
#pragma unroll
            for (int b = 0; b < 8; b += 2) {
                if (a < 2) issue(t + 1, 8 + a * 4 + b / 2);
                Q_FENCE;
                mma(a, b);
                mma(a, b + 1);
                Q_FENCE;
            }
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        Q_FENCE;
    }
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        mma(6, b);
        mma(7, b);
    }
#undef Q_FENCE
    // each wavefront transposes its own part through LDS; one rounding from fp32 (behind the last barrier nobody reads the buffers, and every load
    // into them has landed)
    u16* Es = reinterpret_cast<u16*>(lds) + wave * (128 * QE_LD);
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int b = 0; b < 8; ++b)
            *reinterpret_cast<uint2*>(Es + (a * 16 + l16) * QE_LD + b * 16 + g4 * 4) = make_uint2(pack2hw(acc[a][b][0], acc[a][b][1]), pack2hw(acc[a][b][2], acc[a][b][3]));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 8
    for (int it = 0; it < 32; ++it) {
        const int rr = it * 4 + (lane >> 4), c = l16 * 8, row = m0 + wm * 128 + rr, col = n0 + wn * 128 + c;
        if (row >= g.M || col >= g.N) continue;
        store16((u16*)g.C + (int64_t)row * g.ldc + col, *reinterpret_cast<const uint4*>(Es + rr * QE_LD + c), g.N - col);
    }
}

// A wavefront's WB x WB blocks of 16 x 16, from the lane's first row and first of four columns; one rounding from fp32.
template <typename T, int WB> __device__ __forceinline__ void store_blocks(const QGemmArgs& g, const f32x4 (&acc)[WB][WB], int row0, int col0) {
#pragma unroll
    for (int a = 0; a < WB; ++a) {
        const int row = row0 + a * 16;
        if (row >= g.M) continue;
#pragma unroll
        for (int b = 0; b < WB; ++b) {
            const int col = col0 + b * 16;
            T* dst = (T*)g.C + (int64_t)row * g.ldc + col;
            T v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = from_f32<T>(acc[a][b][i]);
            if (col + 4 <= g.N) {
                __builtin_memcpy(dst, v, sizeof(v));
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (col + i < g.N) dst[i] = v[i];
            }
        }
    }
}

// Products with few output tiles: 32 WB x 32 WB outputs a work group of four wavefronts (2 x 2), each WB x WB blocks of 16 x 16.
// A group is 4 / WB steps (128 bytes of either operand's rows each, as above) and the words with its scales; direct loads fill a ring of NG
// groups.  Behind a group's barrier a wavefront reads the next group's fragments while it multiplies those that it holds, so that a barrier finds
// the group read by everybody, and its place is loaded again.  The sums are those of the large kernel: one chain over the steps, whatever the
// tile.
template <typename T, int WB, int NG>
__global__ __launch_bounds__(256) void quant_ring_kernel(QGemmArgs g) {
    constexpr int SIDE = 32 * WB, TILE = SIDE * 128, G = 4 / WB, GROUP = G * 2 * TILE + 4 * 512;
    constexpr int NL = SIDE / 32, LG = G * 2 * NL + 2;                  // loads of 1 KB per wavefront, operand and step; loads per group
    static_assert(NG * GROUP <= 163840 && LG * (NG - 1) <= 63, "the ring fits the LDS, its loads the counter");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NG * GROUP];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, g4 = lane >> 4;
    int tm, tn;
    if (!tile_of(g, tm, tn)) return;
    const int m0 = tm * SIDE, n0 = tn * SIDE;
    f32x4 acc[WB][WB];
#pragma unroll
    for (int a = 0; a < WB; ++a)
#pragma unroll
        for (int b = 0; b < WB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    unsigned oa[NL], ob[NL];
#pragma unroll
    for (int c = 0; c < NL; ++c) {
        const int row = (wave * NL + c) * 8 + (lane >> 3), ch = (lane & 7) ^ (lane >> 3);
        oa[c] = (unsigned)((int64_t)(min(m0 + row, g.M - 1) - m0) * g.kp + ch * 16);
        ob[c] = (unsigned)((int64_t)(min(n0 + row, g.N - 1) - n0) * g.kp + ch * 16);
    }
    const char* baseA = uniform_ptr(g.A + (int64_t)m0 * g.kp);
    const char* baseB = uniform_ptr(g.B + (int64_t)n0 * g.kp);
    // a lane's word of the row scales belongs to its row of the wavefront's 16 WB (the others repeat), that of the weight's to the wavefront's columns
    const unsigned osa = (unsigned)(min(m0 + wm * 16 * WB + lane % (16 * WB), g.M - 1) - m0) * 4u;
    const char* baseSA = uniform_ptr(g.sa + m0);
    const char* baseSB = uniform_ptr(g.sb + min(n0 + wn * 16 * WB, g.N - 1) / kQBlock);
    const unsigned lds0 = (unsigned)(uintptr_t)lds;
    int issued = 0, slot_in = 0;       // step of the next group to load, and the group's place
    auto issue = [&](int c) {          // load c of the group's LG; past the last step it is loaded again (keeps the counts the same)
        const unsigned dst = lds0 + slot_in * GROUP;
        if (c < 2 * G * NL) {
            const int s = c / (2 * NL), k = c % NL;
            const bool second = c % (2 * NL) >= NL;
            const int64_t at = (int64_t)min(issued + s, g.steps - 1) * 128;
            dma16(second ? ob[k] : oa[k], (second ? baseB : baseA) + at, dst + s * 2 * TILE + (second ? TILE : 0) + (wave * NL + k) * 1024);
        } else {
            const int word = min(issued, g.steps - 1) >> 2;
            if (c == LG - 2) dma4(osa, baseSA + (int64_t)word * g.sa_ld * 4, dst + G * 2 * TILE + wave * 512);
            else             dma4(0, baseSB + (int64_t)word * g.sb_ld * 4, dst + G * 2 * TILE + wave * 512 + 256);
        }
        if (c == LG - 1) {
            issued += G;
            slot_in = slot_in + 1 == NG ? 0 : slot_in + 1;
        }
    };
    const int x0 = (g4 ^ (l16 & 7)) << 4, x1 = ((4 + g4) ^ (l16 & 7)) << 4;
    const int rowA = (wm * 16 * WB + l16) * 128, rowB = (wn * 16 * WB + l16) * 128 + TILE;
    const int scaleA = G * 2 * TILE + wave * 512 + l16 * 4, scaleB = G * 2 * TILE + wave * 512 + 256;
    i32x8 fa[2][G][WB], fb[2][G][WB];
    uint32_t sa[2][WB], sb[2];
    int slot = 0;                      // place of the group whose fragments are read next
    constexpr int NF = 2 * G * WB, NM = G * WB * WB;      // fragments and matrix instructions of a group
    auto read_scales = [&](int set) {
        const unsigned char* st = lds + slot * GROUP;
        sb[set] = *reinterpret_cast<const uint32_t*>(st + scaleB);
#pragma unroll
        for (int a = 0; a < WB; ++a) sa[set][a] = *reinterpret_cast<const uint32_t*>(st + scaleA + a * 64);
    };
    auto read = [&](int f, int set) {  // fragment f of the group's NF
        const unsigned char* st = lds + slot * GROUP;
        const int s = f / (2 * WB), k = f % WB;
        const bool second = f % (2 * WB) < WB;
        const unsigned char* at = st + s * 2 * TILE + (second ? rowB : rowA) + k * 16 * 128;
        const i32x8 v = __builtin_shufflevector(*reinterpret_cast<const i32x4*>(at + x0), *reinterpret_cast<const i32x4*>(at + x1), 0, 1, 2, 3, 4, 5, 6, 7);
        if (second) fb[set][s][k] = v; else fa[set][s][k] = v;
    };
#define Q_FENCE __builtin_amdgcn_sched_barrier(0)
    // with a ring of two groups the loads have half the time, and all of them follow the first instructions
    constexpr int RATE = NG == 2 ? 4 : 1;
    // the group that starts at step t: its matrix instructions, the next group's reads and the last one's loads take turns (loads one behind the other
    // would fill the memory pipeline's queue and hold everything behind them up)
    auto body = [&](int t, auto set_) {
        constexpr int set = decltype(set_)::value;
        // the next group has landed, and every wavefront holds this one's fragments
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LG * (NG - 2)) : "memory");
        read_scales(set ^ 1);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int m = 0; m < NM; ++m) {
#pragma unroll
                for (int f = m * NF / NM; f < (m + 1) * NF / NM; ++f) read(f, set ^ 1);
                Q_FENCE;
                const int s = m / (WB * WB), a = m / WB % WB, b = m % WB, shift = 8 * ((t + s) & 3);
                if (G == 1 || t + s < g.steps) acc[a][b] = q_mma(fb[set][s][b], fa[set][s][a], acc[a][b], sb[set] >> shift, sa[set][a] >> shift);
                Q_FENCE;
#pragma unroll
                for (int c = m * LG * RATE / NM; c < (m + 1) * LG * RATE / NM; ++c)
                    if (c < LG) issue(c);
                Q_FENCE;
            }
        } else {
            constexpr int QM = 4 * G;      // quarters of the group's steps (the rest is better placed by the compiler)
#pragma unroll
            for (int s = 0; s < G; ++s) {
                const int shift = 8 * ((t + s) & 3);
                const float scale_b = __uint_as_float((sb[set] >> shift & 0xffu) << 23);
                float scale_a[WB];
#pragma unroll
                for (int a = 0; a < WB; ++a) scale_a[a] = __uint_as_float((sa[set][a] >> shift & 0xffu) << 23);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const int m = 4 * s + p;
#pragma unroll
                    for (int f = m * NF / QM; f < (m + 1) * NF / QM; ++f) read(f, set ^ 1);
                    if (G == 1 || t + s < g.steps) {
                        bf16x8 x[WB], y[WB];
#pragma unroll
                        for (int k = 0; k < WB; ++k) {
                            x[k] = widened(fb[set][s][k][2 * p], fb[set][s][k][2 * p + 1], scale_b);
                            y[k] = widened(fa[set][s][k][2 * p], fa[set][s][k][2 * p + 1], scale_a[k]);
                        }
#pragma unroll
                        for (int a = 0; a < WB; ++a)
#pragma unroll
                            for (int b = 0; b < WB; ++b) acc[a][b] = mfma16(x[b], y[a], acc[a][b]);
                    }
#pragma unroll
                    for (int c = m * LG * RATE / QM; c < (m + 1) * LG * RATE / QM; ++c)
                        if (c < LG) issue(c);
                }
            }
        }
        slot = slot + 1 == NG ? 0 : slot + 1;
    };
#undef Q_FENCE
#pragma unroll
    for (int u = 0; u < NG; ++u)
#pragma unroll
        for (int c = 0; c < LG; ++c) issue(c);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LG * (NG - 1)) : "memory");
    read_scales(0);
#pragma unroll
    for (int f = 0; f < NF; ++f) read(f, 0);
    slot = 1 % NG;
    for (int t = 0; t < g.steps; t += 2 * G) {
        body(t, std::integral_constant<int, 0>{});
        if (t + G < g.steps) body(t + G, std::integral_constant<int, 1>{});
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the work group's LDS is not handed on with loads on their way to it
    store_blocks<T, WB>(g, acc, m0 + wm * 16 * WB + l16, n0 + wn * 16 * WB + 4 * g4);
}

// fp32 plans, large products: 128 x 128 outputs as above, with two buffers of a step and no fragments held ahead, so that two work groups share a CU and a
// SIMD has two wavefronts to choose from: with the bytes to widen this is a matter of issuing instructions.  4096 x 4096 x 4096 109 us (1.26 PFLOP/s; a
// library product of bf16 operands 1.2); 121 with outputs of 64 bytes a row and store, 148 with a ring of four, one work group a CU.
__global__ __launch_bounds__(256, 2) void quant_f32_kernel(QGemmArgs g) {
    constexpr int WB = 4, SIDE = 32 * WB, TILE = SIDE * 128, NL = SIDE / 32;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * 2 * TILE];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, g4 = lane >> 4;
    int tm, tn;
    if (!tile_of(g, tm, tn)) return;
    const int m0 = tm * SIDE, n0 = tn * SIDE;
    f32x4 acc[WB][WB];
#pragma unroll
    for (int a = 0; a < WB; ++a)
#pragma unroll
        for (int b = 0; b < WB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    unsigned oa[NL], ob[NL];
#pragma unroll
    for (int c = 0; c < NL; ++c) {
        const int row = (wave * NL + c) * 8 + (lane >> 3), ch = (lane & 7) ^ (lane >> 3);
        oa[c] = (unsigned)((int64_t)(min(m0 + row, g.M - 1) - m0) * g.kp + ch * 16);
        ob[c] = (unsigned)((int64_t)(min(n0 + row, g.N - 1) - n0) * g.kp + ch * 16);
    }
    const char* baseA = uniform_ptr(g.A + (int64_t)m0 * g.kp);
    const char* baseB = uniform_ptr(g.B + (int64_t)n0 * g.kp);
    const unsigned ldsw = (unsigned)(uintptr_t)lds + wave * NL * 1024;
    // load c of the 2 NL of step `to`; past the last step the last one is loaded again into the buffer that nobody reads
    auto issue = [&](int to, int c) {
        const int64_t at = (int64_t)min(to, g.steps - 1) * 128;
        const unsigned dst = ldsw + (to & 1) * 2 * TILE;
        if (c < NL) dma16(oa[c], baseA + at, dst + c * 1024);
        else        dma16(ob[c - NL], baseB + at, dst + TILE + (c - NL) * 1024);
    };
    // scale words (four steps') of the lane's rows and of the wavefront's columns
    const uint32_t* const wordB = g.sb + min(n0 + wn * 16 * WB, g.N - 1) / kQBlock;
    uint32_t sa[WB], sb = 0, sa_next[WB], sb_next;
    auto load_scales = [&](int word) {
#pragma unroll
        for (int a = 0; a < WB; ++a) sa_next[a] = g.sa[(int64_t)word * g.sa_ld + min(m0 + (wm * WB + a) * 16 + l16, g.M - 1)];
        sb_next = wordB[(int64_t)word * g.sb_ld];
    };
    const int x[2] = {(g4 ^ (l16 & 7)) << 4, ((4 + g4) ^ (l16 & 7)) << 4};
    const int rowA = (wm * 16 * WB + l16) * 128, rowB = (wn * 16 * WB + l16) * 128 + TILE;
    load_scales(0);
#pragma unroll
    for (int c = 0; c < 2 * NL; ++c) issue(0, c);
    for (int t = 0; t < g.steps; ++t) {
        // the step has landed, and nobody reads the other buffer any more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if ((t & 3) == 0) {
#pragma unroll
            for (int a = 0; a < WB; ++a) sa[a] = sa_next[a];
            sb = sb_next;
            if (t + 4 < g.steps) load_scales((t >> 2) + 1);
        }
        const int shift = 8 * (t & 3);
        const float scale_b = __uint_as_float((sb >> shift & 0xffu) << 23);
        float scale_a[WB];
#pragma unroll
        for (int a = 0; a < WB; ++a) scale_a[a] = __uint_as_float((sa[a] >> shift & 0xffu) << 23);
        const unsigned char* st = lds + (t & 1) * 2 * TILE;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            i32x4 fa[WB], fb[WB];
#pragma unroll
            for (int k = 0; k < WB; ++k) {
                fb[k] = *reinterpret_cast<const i32x4*>(st + rowB + k * 16 * 128 + x[half]);
                fa[k] = *reinterpret_cast<const i32x4*>(st + rowA + k * 16 * 128 + x[half]);
            }
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                bf16x8 wa[WB], wb[WB];
#pragma unroll
                for (int k = 0; k < WB; ++k) {
                    wb[k] = widened(fb[k][2 * p], fb[k][2 * p + 1], scale_b);
                    wa[k] = widened(fa[k][2 * p], fa[k][2 * p + 1], scale_a[k]);
                }
#pragma unroll
                for (int a = 0; a < WB; ++a)
#pragma unroll
                    for (int b = 0; b < WB; ++b) acc[a][b] = mfma16(wb[b], wa[a], acc[a][b]);
#pragma unroll
                for (int c = 0; c < NL; ++c)
                    if (half == 0) issue(t + 1, p * NL + c);
            }
        }
    }
    // each wavefront transposes its own part through LDS (chunk x of four columns of row r at x ^ (r & 15)): a store covers 256 bytes of four rows
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    f32x4* const Es = reinterpret_cast<f32x4*>(lds) + wave * (16 * WB * 4 * WB);
#pragma unroll
    for (int a = 0; a < WB; ++a)
#pragma unroll
        for (int b = 0; b < WB; ++b) Es[(a * 16 + l16) * 16 + ((b * 4 + g4) ^ l16)] = acc[a][b];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 4
    for (int it = 0; it < 16; ++it) {
        const int r = it * 4 + g4, row = m0 + wm * 64 + r, col = n0 + wn * 64 + l16 * 4;
        if (row >= g.M || col >= g.N) continue;
        const f32x4 v = Es[r * 16 + (l16 ^ (r & 15))];
        float* const dst = (float*)g.C + (int64_t)row * g.ldc + col;
        if (col + 4 <= g.N) {
            __builtin_memcpy(dst, &v, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (col + i < g.N) dst[i] = v[i];
        }
    }
}

struct QuantRows {
    uint8_t* Q;
    uint32_t* scales;
    int64_t rows_padded, bytes;
};
static QuantRows quant_rows(int64_t T, int64_t K, void* ws) {
    QuantRows r;
    r.rows_padded = (T + 255) & ~int64_t(255);
    r.Q = (uint8_t*)ws;
    const int64_t q = q_align(T * q_blocks(K) * kQBlock);
    r.scales = (uint32_t*)((uint8_t*)ws + q);
    r.bytes = q + q_align(4 * q_words(K) * r.rows_padded);
    return r;
}

constexpr int64_t kMaxQuantWidth = int64_t(1) << 22;      // 256 rows of a tile are addressed with 32-bit offsets

// Kernel of a product, by the time that a fit of measured times gives it: rounds of work groups, each a fixed part and a part a step; a step takes longer
// the more of the chip is at work.  us, bf16, activations to 8 bits included, chosen / next best, tokens x k x n (weights from HBM):
//   32 x 32, a work group per CU: 8 x 14336 x 4096  15.6 / 22.5, 64 x 4096 x 4096  9.5 / 12.5; two per CU (half the ring): 8 x 4096 x 14336  15.0 / 14.1
//   64 x 64, one: 64 x 4096 x 14336  15.2 / 21.4, 256 x 4096 x 4096  14.3 / 20.8; two: 512 x 4096 x 4096  19.8 / 22.7, 1500 x 2048 x 1001  14.8 / 16.6
//   128 x 128, one: 1024 x 4096 x 4096  25.7 / 33.8, 700 x 14336 x 4096  66 / 91, 300 x 768 x 8192  12.2 / 13.0; two: 2048 x 4096 x 4096  44.1 / 47.2
//   256 x 256: 1024 x 4096 x 14336  51.5 / 84.4, 4096 x 4096 x 4096  63.6 / 85
// fp32: 32 x 32  64 x 4096 x 4096 12.8 / 17.6 (kernel alone), 64 x 64  512 x 4096 x 4096 28.6 / 38.5, 128 x 128  2048 x 4096 x 4096 58.9 / 95.1; one work group per
// CU is never better there.  The bits of a result do not depend on the choice.
struct QuantKernel {
    int side, per_cu;             // outputs of a tile squared; work groups per CU
    double fixed, idle, busy;     // us a round; us a step with one work group on the chip, with one (two) per CU
};
static const QuantKernel kQuantBf16[] = {{32, 1, 1.5, 0.09, 0.13}, {32, 2, 1.5, 0.16, 0.21}, {64, 1, 1.5, 0.19, 0.27}, {64, 2, 2.0, 0.30, 0.42},
                                         {128, 1, 2.0, 0.38, 0.60}, {128, 2, 2.5, 0.60, 1.10}, {256, 1, 4.0, 1.05, 1.50}};
static const QuantKernel kQuantF32[] = {{32, 2, 2.0, 0.21, 0.27}, {64, 2, 3.0, 0.32, 0.64}, {128, 2, 5.5, 0.64, 1.55}};
static int quant_kernel(int64_t M, int64_t N, int64_t steps, int num_cus, const QuantKernel* kernels, int count) {
    int best = 0;
    double best_us = 0;
    for (int i = 0; i < count; ++i) {
        const QuantKernel& k = kernels[i];
        const double tiles = (double)((M + k.side - 1) / k.side) * (double)((N + k.side - 1) / k.side), room = (double)num_cus * k.per_cu;
        const double us = std::ceil(tiles / room) * (k.fixed + (double)steps * (k.idle + (k.busy - k.idle) * std::min(1.0, tiles / room)));
        if (i == 0 || us < best_us) { best = i; best_us = us; }
    }
    return best;
}

template <typename T>
static int quant_product(mlora_plan* p, const void* X, int64_t K, int64_t N, const uint8_t* B, const uint32_t* sb, void* C, void* ws, int kernel,
                         hipStream_t st) {
    const int64_t rows = p->T, kp = q_blocks(K) * kQBlock;
    const QuantRows q = quant_rows(rows, K, ws);
    const int64_t words = q_words(K);
    {
        ProfScope prof(p, MLORA_K_QUANT_ROWS, st);
        const bool few = rows * words < 128 * (int64_t)p->num_cus, past = rows * K * (int64_t)sizeof(T) > int64_t(192) << 20;
        const auto kernel = few ? quant_rows_kernel<T, 1, false> : past ? quant_rows_kernel<T, 8, true> : quant_rows_kernel<T, 8, false>;
        const int64_t per_group = few ? 1 : 8;
        for (int64_t first = 0; first < rows; first += kMaxLaunchGroups * per_group) {
            const int64_t count = std::min(kMaxLaunchGroups * per_group, rows - first);
            const dim3 grid((unsigned)((count + per_group - 1) / per_group), (unsigned)((words + 3) / 4));
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, (const T*)X + first * K, count, K, kp, q.Q + first * kp, q.scales + first, q.rows_padded, (int32_t)words);
        }
    }
    QGemmArgs g{};
    g.A = q.Q; g.sa = q.scales; g.sa_ld = q.rows_padded;
    g.B = B; g.sb = sb; g.sb_ld = q_blocks(N);
    g.C = C; g.ldc = N; g.M = (int32_t)rows; g.N = (int32_t)N; g.steps = (int32_t)q_blocks(K); g.kp = kp;
    constexpr bool F32 = sizeof(T) == 4;
    const QuantKernel* const kernels = F32 ? kQuantF32 : kQuantBf16;
    const int kind = quant_kernel(rows, N, g.steps, p->num_cus, kernels, F32 ? 3 : 7);
    const int64_t side = kernels[kind].side, tiles_m = (rows + side - 1) / side, tiles_n = (N + side - 1) / side, tiles = tiles_m * tiles_n;
    if (tiles > 2 * kMaxLaunchGroups - 256) {      // (2^24 work groups of 256: more outputs than the card holds)
        set_error("8-bit product: too many output tiles");
        return MLORA_ERR_SHAPE;
    }
    g.tiles_m = (int32_t)tiles_m; g.tiles_n = (int32_t)tiles_n;
    g.xcd_run = tiles < 256 ? (int32_t)((tiles + 7) / 8) : 0;
    ProfScope prof(p, kernel, st);
    const dim3 grid((unsigned)(g.xcd_run ? 8 * g.xcd_run : (tiles + 255) / 256 * 256));
    if constexpr (F32) {
        if (kind == 0)      hipLaunchKernelGGL((quant_ring_kernel<T, 1, 2>), grid, dim3(256), 0, st, g);
        else if (kind == 1) hipLaunchKernelGGL((quant_ring_kernel<T, 2, 2>), grid, dim3(256), 0, st, g);
        else                hipLaunchKernelGGL(quant_f32_kernel, grid, dim3(256), 0, st, g);
    } else {
        if (kind == 0)      hipLaunchKernelGGL((quant_ring_kernel<T, 1, 4>), grid, dim3(256), 0, st, g);
        else if (kind == 1) hipLaunchKernelGGL((quant_ring_kernel<T, 1, 2>), grid, dim3(256), 0, st, g);
        else if (kind == 2) hipLaunchKernelGGL((quant_ring_kernel<T, 2, 4>), grid, dim3(256), 0, st, g);
        else if (kind == 3) hipLaunchKernelGGL((quant_ring_kernel<T, 2, 2>), grid, dim3(256), 0, st, g);
        else if (kind == 4) hipLaunchKernelGGL((quant_ring_kernel<T, 4, 4>), grid, dim3(256), 0, st, g);
        else if (kind == 5) hipLaunchKernelGGL((quant_ring_kernel<T, 4, 2>), grid, dim3(256), 0, st, g);
        else                hipLaunchKernelGGL(quant_gemm_kernel, grid, dim3(256), 0, st, g);
    }
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}

static bool misaligned16(const void* q) { return ((uintptr_t)q & 15) != 0; }

static int quant_call(mlora_plan* p, const void* in, const void* w8, void* out, void* ws, bool fwd, void* stream) {
    if (!p) { set_error("plan is NULL"); return MLORA_ERR_NULL; }
    if (p->k > kMaxQuantWidth || p->n > kMaxQuantWidth) { set_error("8-bit product: k or n above 4194304"); return MLORA_ERR_SHAPE; }
    if (p->T == 0) return MLORA_OK;
    if (!in || !w8 || !out) { set_error("8-bit product: an input or the output is NULL"); return MLORA_ERR_NULL; }
    if (!ws) { set_error("workspace is NULL"); return MLORA_ERR_WORKSPACE; }
    if (misaligned16(in) || misaligned16(w8) || misaligned16(out) || misaligned16(ws)) {
        set_error("8-bit product: a pointer is not 16-byte aligned");
        return MLORA_ERR_ALIGN;
    }
    const QuantWeight w = quant_weight(p->k, p->n, const_cast<void*>(w8));
    const int64_t K = fwd ? p->k : p->n, N = fwd ? p->n : p->k;
    const uint8_t* B = fwd ? w.fwd : w.bwd;
    const uint32_t* sb = fwd ? w.fwd_scales : w.bwd_scales;
    const int id = fwd ? MLORA_K_QUANT_GEMM_FWD : MLORA_K_QUANT_GEMM_BWD;
    return p->dtype == MLORA_F32 ? quant_product<float>(p, in, K, N, B, sb, out, ws, id, (hipStream_t)stream)
                                 : quant_product<u16>(p, in, K, N, B, sb, out, ws, id, (hipStream_t)stream);
}

}  // namespace mlora

using namespace mlora;

extern "C" size_t multi_lora_quant_bytes(int64_t k, int64_t n) {
    if (k < 1 || n < 1 || k > kMaxQuantWidth || n > kMaxQuantWidth) return 0;
    return (size_t)quant_weight(k, n, nullptr).bytes;
}

extern "C" int multi_lora_quant_weight(int dtype, int64_t k, int64_t n, const void* W, void* w8, void* stream) {
    if (dtype != MLORA_F32 && dtype != MLORA_BF16) { set_error("dtype must be MLORA_F32 or MLORA_BF16"); return MLORA_ERR_DTYPE; }
    if (k < 1 || n < 1 || k > kMaxQuantWidth || n > kMaxQuantWidth) { set_error("8-bit product: k or n outside [1, 4194304]"); return MLORA_ERR_SHAPE; }
    if (!W || !w8) { set_error("W / w8 is NULL"); return MLORA_ERR_NULL; }
    if (misaligned16(W) || misaligned16(w8)) { set_error("W / w8 is not 16-byte aligned"); return MLORA_ERR_ALIGN; }
    const QuantWeight q = quant_weight(k, n, w8);
    const dim3 grid((unsigned)q_blocks(n), (unsigned)q_blocks(k));
    if (dtype == MLORA_F32) hipLaunchKernelGGL(quant_weight_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, (const float*)W, k, n, q);
    else                    hipLaunchKernelGGL(quant_weight_kernel<u16>, grid, dim3(256), 0, (hipStream_t)stream, (const u16*)W, k, n, q);
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}

extern "C" size_t multi_lora_quant_workspace_bytes(const mlora_plan* plan) {
    if (!plan) return 0;
    return (size_t)std::max(quant_rows(plan->T, plan->k, nullptr).bytes, quant_rows(plan->T, plan->n, nullptr).bytes);
}

extern "C" int multi_lora_quant_fwd(mlora_plan* plan, const void* X, const void* w8, void* Y, void* workspace, void* stream) {
    return quant_call(plan, X, w8, Y, workspace, true, stream);
}

extern "C" int multi_lora_quant_bwd(mlora_plan* plan, const void* dY, const void* w8, void* dX, void* workspace, void* stream) {
    return quant_call(plan, dY, w8, dX, workspace, false, stream);
}
