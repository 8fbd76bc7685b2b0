// Block edges: the norm after a block, its gate and residual scale, the residual sum and the norm before the next block, forward
// and backward, per adapter over the segmentation of a plan.
//
//   forward    ry = 1 / sqrt(mean(y^2) + eps_post),  h' = h + s_i g_i w_post (y ry)
//              rh = 1 / sqrt(mean(h'^2) + eps_pre),  x = w_pre (h' rh)
//   backward   with yh = y ry, xh = h' rh, q = g_i w_post (g absent: q = w_post):
//              e  = dh' + rh (w_pre dx - xh mean(w_pre dx xh)),  dh = e
//              dy = s_i ry (q e - yh mean(q e yh))
//              C_i = sum_t e yh,  D_i = sum_t dx xh  over the adapter's rows:  d_gate = s_i w_post C_i,  d_post = s_i g_i C_i,
//              d_pre = D_i,  d_scale = sum_t sum_c q e yh;  gains that all adapters share sum over the adapters
// Bound by memory: 32768 x 8192 bf16 with all gradients, forward 428 us and backward 611 + 18 (5.0 and 5.3 TB/s; a copy 5.2).
// A row is read once: a group of wavefronts holds it in registers between the sums and the outputs.  The backward needs one
// round of sums only: mean(q e yh) follows from the sums of q yh (dh' + rh w_pre dx) and q yh xh and from mean(w_pre dx xh).
// A work group walks a run of consecutive rows with its columns' gains, and in the backward the sums
// C and D of its columns, in registers; where the run passes from one adapter to the next it stores the sums and takes the next
// gains.  Run w of the rows and adapter i meet at most once, and either w or i grows from one meeting to the next: the partial sums
// of a meeting are in slot w + i, and an adapter's slots are consecutive.
#include <algorithm>
#include <cmath>

#include "stream_common.h"

namespace mlora {

struct EdgeArgs {
    int64_t T, d;
    int32_t N, run;                    // adapters; rows of a work group's run
    const int32_t* off;                // [N + 1]
    const void* post; int64_t post_ld; // gains: [d], or a row per adapter (ld > 0)
    const void* gate; int64_t gate_ld;
    const void* pre;  int64_t pre_ld;
    const float* scale;                // [N] or NULL
    float eps_post, eps_pre;
    const void* h; const void* y; void* h_out; void* x; float* stats;            // forward; stats: ry[T], rh[T]
    const void* dx; const void* dh_out; void* dh; void* dy;                      // backward (reads h, y, stats)
    float* partC; float* partD; float* partS;                                    // [slots][d], [slots][d], [slots]
    bool past;                         // forward: the rows do not fit three quarters of the Infinity Cache, and its outputs go past it
};

// A forward's output; past the caches (bf16, whole pieces) where `past` (uniform) says so: 16384 x 4096 108 -> 85 us.  (The backward gains 1 % where its
// registers allow it, and the choice costs it 9 %.)
template <typename T> __device__ __forceinline__ void put_piece(T* p, const Piece<T>& v, int valid, bool past) {
    if (sizeof(T) == 2 && past) store16(p, v.w[0], valid);
    else store_piece(p, v, valid);
}

// Sum of NV values over the W wavefronts of a work group; every lane gets the same bits.  The caller alternates between two pieces of
// LDS: a wavefront that is one sum ahead writes to the other one.
template <int W, int NV> __device__ __forceinline__ void worker_sum(float (&v)[NV], float* red, int wave) {
#pragma unroll
    for (int q = 0; q < NV; ++q) v[q] = wave_sum(v[q]);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int q = 0; q < NV; ++q) red[q * W + wave] = v[q];
        }
        lds_barrier();
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            v[q] = red[q * W];
#pragma unroll
            for (int w = 1; w < W; ++w) v[q] += red[q * W + w];
        }
    }
}

// Index of the adapter that owns row t, by 64 ends at a time: two loads, one after the other, for any number of adapters (one up to 64).
__device__ __forceinline__ int owner_of_row(const int32_t* off, int N, int64_t t) {
    static_assert(MLORA_MAX_ADAPTERS <= 64 * 64, "two rounds");
    const int lane = threadIdx.x & 63, stride = (N + 63) >> 6;
    auto ended = [&](int first, int step, int count) {      // of the adapters first + step - 1, first + 2 step - 1, ...: how many end at or before t
        const int end = first + (lane + 1) * step;
        return (int)__popcll(__ballot(lane < count && end <= N && off[min(end, N)] <= t));
    };
    const int i = ended(0, stride, 64) * stride;
    return stride == 1 ? i : i + ended(i, 1, stride);
}

enum { kPieces, kAny, kNarrow };

// WIDTH: a multiple of eight, so that a piece is whole or absent (the handling of a part costs these kernels a third of their registers
// more); any other; below eight.  W wavefronts share a row, NP pieces of eight columns a lane.  The next row's loads are in flight while a row's sums are
// taken: without them a row's time is a memory latency plus that of the sums.
template <typename T, int W, int NP, bool POST, bool PRE, int WIDTH>
__global__ __launch_bounds__(64 * W) void edge_fwd_kernel(EdgeArgs g) {
    __shared__ float red[2][W];
    constexpr bool AHEAD = NP == 1;    // wider rows leave no registers for it
    constexpr bool FULL = WIDTH == kPieces, whole = WIDTH != kNarrow;
    const int wave = threadIdx.x >> 6;
    const int64_t worker = blockIdx.x, t0 = worker * g.run, t1 = min(g.T, t0 + g.run);
    int64_t next = t0;                 // first row that needs other gains
    float q[NP][kPiece], w[NP][kPiece];
    auto column = [&](int j) { return (j * 64 * W + (int)threadIdx.x) * kPiece; };
    auto valid_at = [&](int c) { return FULL ? ((int)g.d > c ? kPiece : 0) : (int)g.d - c; };
    Piece<T> hn[NP], yn[NP];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int c = column(j), valid = valid_at(c);
            if (valid <= 0) continue;
            hn[j] = load_raw((const T*)g.h + t * g.d + c, valid, whole);
            if (POST) yn[j] = load_raw((const T*)g.y + t * g.d + c, valid, whole);
        }
    };
    if (AHEAD) load(t0);
    int i = owner_of_row(g.off, g.N, t0);
    for (int64_t t = t0; t < t1; ++t) {
        if (t == next) {
            while (g.off[i + 1] <= t) ++i;
            next = g.off[i + 1];
            const float s = POST && g.scale ? g.scale[i] : 1.f;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = column(j), valid = valid_at(c);
                if (valid <= 0) continue;
                if (POST) {
                    unpack(load_piece((const T*)g.post + i * g.post_ld + c, valid, whole), q[j]);
                    float ga[kPiece];
                    if (g.gate) unpack(load_piece((const T*)g.gate + i * g.gate_ld + c, valid, whole), ga);
#pragma unroll
                    for (int k = 0; k < kPiece; ++k) q[j][k] *= g.gate ? s * ga[k] : s;
                }
                if (PRE) unpack(load_piece((const T*)g.pre + i * g.pre_ld + c, valid, whole), w[j]);
            }
        }
        if (!AHEAD) load(t);
        const int64_t row = t * g.d;
        float h[NP][kPiece], y[NP][kPiece];
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int valid = valid_at(column(j));
            if (valid <= 0) continue;
            if (!FULL) settle(hn[j], valid, whole);
            unpack(hn[j], h[j]);
            if (POST) {
                if (!FULL) settle(yn[j], valid, whole);
                unpack(yn[j], y[j]);
#pragma unroll
                for (int k = 0; k < kPiece; ++k) sum[0] += y[j][k] * y[j][k];
            }
        }
        if (AHEAD && t + 1 < t1) load(t + 1);
        if (POST) {
            worker_sum<W, 1>(sum, red[0], wave);
            const float ry = 1.0f / sqrtf(sum[0] / (float)g.d + g.eps_post);
            if (g.stats && threadIdx.x == 0) g.stats[t] = ry;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = column(j), valid = valid_at(c);
                if (valid <= 0) continue;
#pragma unroll
                for (int k = 0; k < kPiece; ++k) h[j][k] += q[j][k] * (y[j][k] * ry);
                put_piece((T*)g.h_out + row + c, pack<T>(h[j]), valid, g.past);
            }
        }
        if (PRE) {       // the norm takes the sum as it is in registers, not its rounding to the stored type
            sum[0] = 0.f;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                if (valid_at(column(j)) <= 0) continue;
#pragma unroll
                for (int k = 0; k < kPiece; ++k) sum[0] += h[j][k] * h[j][k];      // columns past d are zeros
            }
            worker_sum<W, 1>(sum, red[1], wave);
            const float rh = 1.0f / sqrtf(sum[0] / (float)g.d + g.eps_pre);
            if (g.stats && threadIdx.x == 0) g.stats[g.T + t] = rh;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = column(j), valid = valid_at(c);
                if (valid <= 0) continue;
                float x[kPiece];
#pragma unroll
                for (int k = 0; k < kPiece; ++k) x[k] = w[j][k] * (h[j][k] * rh);
                put_piece((T*)g.x + row + c, pack<T>(x), valid, g.past);
            }
        }
        if (W > 1 && POST != PRE) lds_barrier();      // one sum a row: its LDS is free before the next row's
    }
}

// G: rows that a work group has in hand at a time, W wavefronts each (G > 1 for rows of one wavefront only: their sums need no barrier).  The sums C and D
// of the G rows' wavefronts are added through LDS where an adapter's rows of the run end.  Rows of more than a piece a lane (NP > 1) leave no
// registers for the next row, and where they take sixteen wavefronts none for the row behind its sums: its tensors are read again, from the L2.
// Four wavefronts a SIMD for bf16 rows of several wavefronts, where odd widths would take a few registers more: 20000 x 2697 with gradients 181 us, 203 without (fp32 spills
// more: 292 against 281).
template <typename T, int W, int NP, int G, bool POST, bool PRE, int WIDTH>
__global__ __launch_bounds__(64 * W * G, sizeof(T) == 2 && G == 1 ? 4 : 1) void edge_bwd_kernel(EdgeArgs g) {
    static_assert(G == 1 || W == 1, "barriers of a row's sums are the work group's");
    constexpr bool AHEAD = NP == 1, AGAIN = NP > 1 && G == 1, FULL = WIDTH == kPieces, whole = WIDTH != kNarrow;
    __shared__ float red[2][3 * W];
    __shared__ f32x4 parts[G > 1 ? 2 : 1][G > 1 ? G : 1][G > 1 ? 128 * NP : 1];      // [C, D][row][half a piece of a lane]
    __shared__ float partS[G];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = G > 1 ? wave : 0;
    const int64_t worker = blockIdx.x, t0 = worker * g.run, t1 = min(g.T, t0 + g.run);
    int i = 0;
    float s = 1.f, accS = 0.f;
    float q[NP][kPiece], w[NP][kPiece], C[NP][kPiece], D[NP][kPiece];
    auto column = [&](int j) { return (j * 64 * W + (G > 1 ? lane : (int)threadIdx.x)) * kPiece; };
    auto valid_at = [&](int c) { return FULL ? ((int)g.d > c ? kPiece : 0) : (int)g.d - c; };
    // sums of the run's rows of adapter i
    auto flush = [&]() {
        const int64_t slot = (worker + i) * g.d;
        if constexpr (G > 1) {
#pragma unroll
            for (int j = 0; j < NP; ++j)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float (&v)[kPiece] = x ? D[j] : C[j];
                    parts[x][group][128 * j + lane] = f32x4{v[0], v[1], v[2], v[3]};
                    parts[x][group][128 * j + 64 + lane] = f32x4{v[4], v[5], v[6], v[7]};
                }
            if (lane == 0) partS[group] = accS;
            lds_barrier();
            // wavefronts 0, 1 the halves of C, 2, 3 those of D
            static_assert(G == 4, "a wavefront for each half of each sum");
            const int x = wave >> 1;
            float* const out = x ? (PRE ? g.partD : nullptr) : (POST ? g.partC : nullptr);
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = column(j) + 4 * (wave & 1), valid = min(4, valid_at(c));
                if (!out || valid <= 0) continue;
                const int at = 128 * j + (wave & 1) * 64 + lane;
                const f32x4 v = ((parts[x][0][at] + parts[x][1][at]) + parts[x][2][at]) + parts[x][3][at];
                if (valid == 4) {
                    __builtin_memcpy(out + slot + c, &v, 16);
                } else {
#pragma unroll
                    for (int k = 0; k < 3; ++k)
                        if (k < valid) out[slot + c + k] = v[k];
                }
            }
            if (POST && g.partS && threadIdx.x == 0) g.partS[worker + i] = ((partS[0] + partS[1]) + partS[2]) + partS[3];
            lds_barrier();
        } else {
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = column(j), valid = valid_at(c);
                if (valid <= 0) continue;
                if (POST && g.partC) store_piece(g.partC + slot + c, pack<float>(C[j]), valid);
                if (PRE && g.partD) store_piece(g.partD + slot + c, pack<float>(D[j]), valid);
            }
            if (POST && g.partS && threadIdx.x == 0) g.partS[worker + i] = accS;
        }
    };
    struct Raw {
        Piece<T> dh, y, dx, h;
    };
    Raw raw[AHEAD ? NP : 1];
    float ryn = 0.f, rhn = 0.f;
    auto load_stats = [&](int64_t t) {
        if (POST) ryn = g.stats[t];
        if (PRE) rhn = g.stats[g.T + t];
    };
    auto load = [&](Raw& r, int64_t t, int j) {
        const int c = column(j), valid = valid_at(c);
        if (valid <= 0) return;
        const int64_t at = t * g.d + c;
        if (POST) r.y = load_raw((const T*)g.y + at, valid, whole);
        if (PRE) {
            r.h = load_raw((const T*)g.h + at, valid, whole);
            r.dx = load_raw((const T*)g.dx + at, valid, whole);
        }
        if (g.dh_out) r.dh = load_raw((const T*)g.dh_out + at, valid, whole);
    };
    // yh, xh and e = dh' + rh w dx (the mean is taken off later) of a piece
    auto form = [&](Raw& r, int j, float ry, float rh, float (&e)[kPiece], float (&yh)[kPiece], float (&xh)[kPiece], float (&u)[kPiece], float (&dx)[kPiece]) {
        const int valid = valid_at(column(j));
        if (!FULL && valid < kPiece) {
            if (g.dh_out) settle(r.dh, valid, whole);
            if (POST) settle(r.y, valid, whole);
            if (PRE) {
                settle(r.h, valid, whole);
                settle(r.dx, valid, whole);
            }
        }
        if (g.dh_out) {
            unpack(r.dh, e);
        } else {
#pragma unroll
            for (int k = 0; k < kPiece; ++k) e[k] = 0.f;
        }
        if (POST) {
            unpack(r.y, yh);
#pragma unroll
            for (int k = 0; k < kPiece; ++k) {
                yh[k] *= ry;
                u[k] = q[j][k] * yh[k];
            }
        }
        if (PRE) {
            unpack(r.dx, dx);
            unpack(r.h, xh);
#pragma unroll
            for (int k = 0; k < kPiece; ++k) {
                if (POST) xh[k] += s * u[k];      // h', not rounded to the stored type
                xh[k] *= rh;
                e[k] += rh * (w[j][k] * dx[k]);
            }
        }
    };
    auto load_all = [&](int64_t t) {
        load_stats(t);
#pragma unroll
        for (int j = 0; j < (AHEAD ? NP : 0); ++j) load(raw[j], t, j);
    };
    if (AHEAD && t0 + group < t1) load_all(t0 + group);
    i = owner_of_row(g.off, g.N, t0);
    for (int64_t begin = t0; begin < t1;) {        // the run's rows of one adapter after the other
        while (g.off[i + 1] <= begin) ++i;
        const int64_t end = min(t1, (int64_t)g.off[i + 1]);
        s = POST && g.scale ? g.scale[i] : 1.f;
        accS = 0.f;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
#pragma unroll
            for (int k = 0; k < kPiece; ++k) { C[j][k] = 0.f; D[j][k] = 0.f; }
            const int c = column(j), valid = valid_at(c);
            if (valid <= 0) continue;
            if (POST) {
                unpack(load_piece((const T*)g.post + i * g.post_ld + c, valid, whole), q[j]);
                if (g.gate) {
                    float ga[kPiece];
                    unpack(load_piece((const T*)g.gate + i * g.gate_ld + c, valid, whole), ga);
#pragma unroll
                    for (int k = 0; k < kPiece; ++k) q[j][k] *= ga[k];
                }
            }
            if (PRE) unpack(load_piece((const T*)g.pre + i * g.pre_ld + c, valid, whole), w[j]);
        }
        // the wavefronts' rows go round from the start of the run
        for (int64_t t = begin + (G > 1 ? (group - (begin - t0) % G + G) % G : 0); t < end; t += G) {
            if (!AHEAD) load_stats(t);
            const int64_t row = t * g.d;
            const float ry = ryn, rh = rhn;
            float e[NP][kPiece], yh[NP][kPiece], xh[NP][kPiece], u[kPiece], dx[kPiece];
            float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                if (valid_at(column(j)) <= 0) continue;
                Raw& r = raw[AHEAD ? j : 0];
                if (!AHEAD) load(r, t, j);
                form(r, j, ry, rh, e[j], yh[j], xh[j], u, dx);
#pragma unroll
                for (int k = 0; k < kPiece; ++k) {
                    if (PRE) {
                        D[j][k] += dx[k] * xh[j][k];
                        sum[0] += w[j][k] * dx[k] * xh[j][k];
                    }
                    if (POST) {
                        sum[1] += u[k] * e[j][k];
                        if (PRE) sum[2] += u[k] * xh[j][k];
                    }
                }
            }
            if (AHEAD && t + G < t1) load_all(t + G);
            worker_sum<W, 3>(sum, red[(t - t0) & 1], wave);
            const float inv_d = 1.0f / (float)g.d;
            const float m1 = PRE ? rh * sum[0] * inv_d : 0.f;
            const float dot = sum[1] - m1 * sum[2];       // sum over the columns of q e yh
            const float m2 = dot * inv_d;
            accS += dot;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = column(j), valid = valid_at(c);
                if (valid <= 0) continue;
                if (AGAIN) {
                    load(raw[0], t, j);
                    form(raw[0], j, ry, rh, e[j], yh[j], xh[j], u, dx);
                }
                float dy[kPiece];
#pragma unroll
                for (int k = 0; k < kPiece; ++k) {
                    if (PRE) e[j][k] -= m1 * xh[j][k];
                    if (POST) {
                        C[j][k] += e[j][k] * yh[j][k];
                        dy[k] = s * ry * (q[j][k] * e[j][k] - yh[j][k] * m2);
                    }
                }
                store_piece((T*)g.dh + row + c, pack<T>(e[j]), valid);
                if (POST) store_piece((T*)g.dy + row + c, pack<T>(dy), valid);
            }
        }
        flush();
        begin = end;
    }
}

// Sums of an adapter's slots, in the order of the rows, and the gradients that belong to one adapter.  Gains that the adapters share
// leave the adapter's sum in its first slot for edge_shared_kernel.  blockIdx.y = adapter.
struct EdgeReduceArgs {
    int64_t d;
    int32_t N, run;
    const int32_t* off;
    const void* post; int64_t post_ld;
    const void* gate; int64_t gate_ld;
    const float* scale;
    float* partC; float* partD; float* partS;
    void* d_post; void* d_gate; void* d_pre; float* d_scale;
    int64_t pre_ld;
    int32_t accum;
};

template <typename T> __device__ __forceinline__ void put_gradient(void* out, int64_t at, float v, int accum) {
    T* p = (T*)out + at;
    *p = from_f32<T>(accum ? to_f32<T>(*p) + v : v);
}

// slots of adapter i: [first, last]; none if it has no rows
__device__ __forceinline__ bool adapter_slots(const int32_t* off, int i, int run, int64_t& first, int64_t& last) {
    const int32_t a = off[i], b = off[i + 1];
    if (a >= b) return false;
    first = a / run + i;
    last = (b - 1) / run + i;
    return true;
}

// A work group takes 64 columns, sixteen lanes of four columns: lane group s adds the slots first + s, first + s + 32, ..., and the 32 sums are added in
// that order.
template <typename T>
__global__ __launch_bounds__(512) void edge_reduce_kernel(EdgeReduceArgs g) {
    __shared__ float sums[2][32][64];
    const int i = blockIdx.y, tid = threadIdx.x, group = tid >> 4, c4 = (tid & 15) * 4;
    const int64_t c0 = (int64_t)blockIdx.x * 64;
    const int valid = (int)min((int64_t)4, g.d - c0 - c4);
    int64_t first = 0, last = -1;
    const bool any = adapter_slots(g.off, i, g.run, first, last);
    const int64_t c = c0 + (tid & 63);
    float s = 1.f, w = 0.f, ga = 1.f, S = 0.f;              // on their way with the sums
    if (g.d_scale && blockIdx.x == 0 && first + tid <= last) S = g.partS[first + tid];
    if (any && tid < 64 && c < g.d && (g.d_gate || g.d_post)) {      // (an adapter without rows has zeros whatever its parameters hold)
        if (g.scale) s = g.scale[i];
        w = to_f32<T>(((const T*)g.post)[i * g.post_ld + c]);
        if (g.gate) ga = to_f32<T>(((const T*)g.gate)[i * g.gate_ld + c]);
    }
    f32x4 C = {0.f, 0.f, 0.f, 0.f}, D = C;
    if (valid > 0) {
#pragma unroll 4
        for (int64_t k = first + group; k <= last; k += 32) {
            const int64_t at = k * g.d + c0 + c4;
            if (g.partC) C += __builtin_bit_cast(f32x4, load16(g.partC + at, valid));
            if (g.partD) D += __builtin_bit_cast(f32x4, load16(g.partD + at, valid));
        }
    }
    *reinterpret_cast<f32x4*>(&sums[0][group][c4]) = C;
    *reinterpret_cast<f32x4*>(&sums[1][group][c4]) = D;
    if (g.d_scale && blockIdx.x == 0) {
        float v = S;
        for (int64_t k = first + tid + 512; k <= last; k += 512) v += g.partS[k];
        v = wave_sum(v);
        __shared__ float waves[8];
        if ((tid & 63) == 0) waves[tid >> 6] = v;
        __syncthreads();
        if (tid == 0) {
            v = waves[0];
            for (int w = 1; w < 8; ++w) v += waves[w];
            g.d_scale[i] = g.accum ? g.d_scale[i] + v : v;
        }
    }
    __syncthreads();
    if (tid >= 128 || c >= g.d) return;
    float v = sums[tid >> 6][0][tid & 63];
#pragma unroll
    for (int k = 1; k < 32; ++k) v += sums[tid >> 6][k][tid & 63];
    if (tid < 64) {
        if (g.d_gate && g.gate_ld) put_gradient<T>(g.d_gate, i * g.gate_ld + c, s * w * v, g.accum);
        if (g.d_post && g.post_ld) put_gradient<T>(g.d_post, i * g.post_ld + c, s * ga * v, g.accum);
        if (any && g.partC) g.partC[first * g.d + c] = v;
    } else {
        if (g.d_pre && g.pre_ld) put_gradient<T>(g.d_pre, i * g.pre_ld + c, v, g.accum);
        if (any && g.partD) g.partD[first * g.d + c] = v;
    }
}

// Gradients of the gains that all adapters share: a work group takes 64 columns, wavefront v the adapters v, v + 4, ...; the four sums are added in
// that order.
template <typename T>
__global__ __launch_bounds__(256) void edge_shared_kernel(EdgeReduceArgs g) {
    __shared__ int64_t slot[256];
    __shared__ float scale[256], sums[3][4][64];
    const int tid = threadIdx.x, wave = tid >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + (tid & 63);
    float gate = 0.f, post = 0.f, pre = 0.f;
    const float w0 = g.post && !g.post_ld && c < g.d ? to_f32<T>(((const T*)g.post)[c]) : 0.f;
    const float g0 = g.gate && !g.gate_ld && c < g.d ? to_f32<T>(((const T*)g.gate)[c]) : 1.f;
    for (int base = 0; base < g.N; base += 256) {
        const int count = min(256, g.N - base);
        __syncthreads();
        if (tid < count) {
            int64_t first, last;
            slot[tid] = adapter_slots(g.off, base + tid, g.run, first, last) ? first : -1;
            scale[tid] = g.scale ? g.scale[base + tid] : 1.f;
        }
        __syncthreads();
        if (c >= g.d) continue;
#pragma unroll 4
        for (int k = wave; k < count; k += 4) {
            const int i = base + k;
            if (slot[k] < 0) continue;
            if (g.partC) {
                const float C = scale[k] * g.partC[slot[k] * g.d + c];
                gate += (g.post_ld ? to_f32<T>(((const T*)g.post)[i * g.post_ld + c]) : w0) * C;
                post += (g.gate && g.gate_ld ? to_f32<T>(((const T*)g.gate)[i * g.gate_ld + c]) : g0) * C;
            }
            if (g.partD) pre += g.partD[slot[k] * g.d + c];
        }
    }
    sums[0][wave][tid & 63] = gate;
    sums[1][wave][tid & 63] = post;
    sums[2][wave][tid & 63] = pre;
    __syncthreads();
    if (c >= g.d || wave == 3) return;
    const float (&v)[4][64] = sums[wave];
    const float total = ((v[0][tid & 63] + v[1][tid & 63]) + v[2][tid & 63]) + v[3][tid & 63];
    void* const out = wave == 0 ? (g.gate_ld ? nullptr : g.d_gate) : wave == 1 ? (g.post_ld ? nullptr : g.d_post) : (g.pre_ld ? nullptr : g.d_pre);
    if (out) put_gradient<T>(out, c, total, g.accum);
}

// Rows that are on the chip at a time, with sixteen wavefronts a CU.
static int64_t edge_resident(const mlora_plan* p, int64_t d) {
    int64_t waves = 1;
    while (waves < 16 && waves * 64 * kPiece < d) waves *= 2;
    return p->num_cus * (16 / waves);
}
static int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Rows that a backward's work group has in hand: four, a wavefront each, where a wavefront's lanes hold a row in a piece, or in two and there are rows for
// sixteen a CU (four rows share a run's partial sums, and each wavefront loads the gains).  Two wavefronts a row / four rows, us with gradients, T x d:
// 4096 x 1001 fp32 46.7 / 44.1, 8192 x 1024 bf16 43.9 / 35.1, 8192 x 1001 fp32 87.3 / 65.8; but 3000 x 1024 fp32 25.4 / 27.2, 2048 x 1024 bf16 15.4 / 17.4.
static int64_t edge_groups(int64_t T, int64_t d, int num_cus) { return d <= 64 * kPiece || (d <= 128 * kPiece && T >= 16 * (int64_t)num_cus) ? 4 : 1; }
// Rows of a backward's run: one round of work groups, so that there are few partial sums (8 d bytes a run, written and read again); four rows at least
// where that leaves a work group per CU.
static int32_t edge_run(const mlora_plan* p, int64_t d) {
    const int64_t rows = edge_groups(p->T, d, p->num_cus);      // rows that a work group has in hand
    const int64_t resident = d <= 64 * kPiece ? 12 * (int64_t)p->num_cus : edge_resident(p, d);      // (three work groups a CU, by their registers)
    return (int32_t)std::max(rows * div_up(p->T, resident), std::min<int64_t>(4, div_up(p->T, p->num_cus)));
}
// Rows of a forward's run, which only saves the gains' loads; more where a launch (fewer than 2^32 work items, up to 1024 a work group) has no room for so many.
static int32_t edge_run_forward(const mlora_plan* p, int64_t d) {
    return (int32_t)std::max(std::min<int64_t>(8, div_up(p->T, edge_resident(p, d))), div_up(p->T, (int64_t(1) << 22) - 1));
}
static int64_t edge_slots(const mlora_plan* p, int64_t d) { return p->T == 0 ? 0 : div_up(p->T, edge_run(p, d)) + p->N; }

constexpr int64_t kMaxEdgeCols = 8 * 64 * 4 * kPiece;      // a row in the registers of eight wavefronts

static int check_edge(const mlora_plan* p, const mlora_edge* e) {
    if (!p || !e) { set_error("plan / edge is NULL"); return MLORA_ERR_NULL; }
    if (p->N == 0) { set_error("block edge: the plan has no adapters"); return MLORA_ERR_SHAPE; }
    if (e->d < 1 || e->d > kMaxEdgeCols) { set_error("block edge: the width is outside [1, MLORA_MAX_EDGE_WIDTH]"); return MLORA_ERR_SHAPE; }
    if (!e->post_gain && !e->pre_gain) { set_error("block edge: neither post_gain nor pre_gain is given"); return MLORA_ERR_NULL; }
    if (!e->post_gain && (e->gate || e->res_scale)) { set_error("block edge: gate and res_scale belong to post_gain, which is NULL"); return MLORA_ERR_NULL; }
    for (int64_t ld : {e->post_ld, e->gate_ld, e->pre_ld})
        if (ld != 0 && ld < e->d) { set_error("block edge: a gain's row stride is neither 0 nor at least the width"); return MLORA_ERR_SHAPE; }
    if ((e->post_gain && !(e->post_eps > 0.f && std::isfinite(e->post_eps))) || (e->pre_gain && !(e->pre_eps > 0.f && std::isfinite(e->pre_eps)))) {
        set_error("block edge: eps is not positive and finite");
        return MLORA_ERR_SCALE;
    }
    return MLORA_OK;
}

static int check_element_aligned(const mlora_plan* p, std::initializer_list<const void*> elems, std::initializer_list<const void*> floats) {
    const uintptr_t es = p->dtype == MLORA_F32 ? 4 : 2;
    for (const void* q : elems)
        if ((uintptr_t)q & (es - 1)) { set_error("block edge: a tensor is not aligned to its elements"); return MLORA_ERR_ALIGN; }
    for (const void* q : floats)
        if ((uintptr_t)q & 3) { set_error("block edge: res_scale, stats, d_scale or workspace is not 4-byte aligned"); return MLORA_ERR_ALIGN; }
    return MLORA_OK;
}

template <typename T, bool POST, bool PRE, int WIDTH>
static void launch_edge_of_width(const EdgeArgs& g, int num_cus, bool fwd, hipStream_t st) {
    const int64_t workers = (g.T + g.run - 1) / g.run, pieces = (g.d + kPiece - 1) / kPiece;
#define MLORA_EDGE(W, NP, G, WF, NF)                                                                                               \
    do {                                                                                                                           \
        if (fwd) hipLaunchKernelGGL((edge_fwd_kernel<T, WF, NF, POST, PRE, WIDTH>), dim3((unsigned)workers), dim3(64 * WF), 0, st, g);    \
        else     hipLaunchKernelGGL((edge_bwd_kernel<T, W, NP, G, POST, PRE, WIDTH>), dim3((unsigned)workers), dim3(64 * W * G), 0, st, g); \
    } while (0)
    if (WIDTH == kNarrow || pieces <= 64) { MLORA_EDGE(1, 1, 4, 1, 1); return; }
    if constexpr (WIDTH == kNarrow) return;
    else if (pieces <= 128 && edge_groups(g.T, g.d, num_cus) == 4) MLORA_EDGE(1, 2, 4, 2, 1);
    else if (pieces <= 128) MLORA_EDGE(2, 1, 1, 2, 1);
    else if (pieces <= 256) MLORA_EDGE(4, 1, 1, 4, 1);
    else if (pieces <= 512) MLORA_EDGE(8, 1, 1, 8, 1);
    else if (pieces <= 1024) MLORA_EDGE(16, 1, 1, 16, 1);
    else MLORA_EDGE(16, 2, 1, 8, 4);
#undef MLORA_EDGE
}
template <typename T, bool POST, bool PRE> static void launch_edge(const EdgeArgs& g, int num_cus, bool fwd, hipStream_t st) {
    if (g.d % kPiece == 0)  launch_edge_of_width<T, POST, PRE, kPieces>(g, num_cus, fwd, st);
    else if (g.d > kPiece)  launch_edge_of_width<T, POST, PRE, kAny>(g, num_cus, fwd, st);
    else                    launch_edge_of_width<T, POST, PRE, kNarrow>(g, num_cus, fwd, st);
}
template <typename T> static void launch_edge(const EdgeArgs& g, int num_cus, bool fwd, hipStream_t st) {
    if (g.post && g.pre) launch_edge<T, true, true>(g, num_cus, fwd, st);
    else if (g.post)     launch_edge<T, true, false>(g, num_cus, fwd, st);
    else                 launch_edge<T, false, true>(g, num_cus, fwd, st);
}

static EdgeArgs edge_args(const mlora_plan* p, const mlora_edge* e) {
    EdgeArgs g{};
    g.T = p->T; g.d = e->d; g.N = p->N; g.off = p->view.off;
    g.post = e->post_gain; g.post_ld = e->post_ld; g.gate = e->gate; g.gate_ld = e->gate_ld; g.pre = e->pre_gain; g.pre_ld = e->pre_ld;
    g.scale = e->res_scale; g.eps_post = e->post_eps; g.eps_pre = e->pre_eps;
    return g;
}

}  // namespace mlora

using namespace mlora;

extern "C" int multi_lora_edge_fwd(mlora_plan* plan, const mlora_edge* edge, const void* h, const void* y, void* h_out, void* x, float* stats,
                                   void* stream) {
    int rc = check_edge(plan, edge);
    if (rc != MLORA_OK) return rc;
    if (plan->T == 0) return MLORA_OK;
    if (!h || (edge->post_gain && (!y || !h_out)) || (edge->pre_gain && !x)) {
        set_error("block edge: h, y, h_out or x is NULL although its norm is given");
        return MLORA_ERR_NULL;
    }
    if ((rc = check_element_aligned(plan, {h, y, h_out, x, edge->post_gain, edge->gate, edge->pre_gain}, {stats, edge->res_scale})) != MLORA_OK) return rc;
    EdgeArgs g = edge_args(plan, edge);
    g.h = h; g.y = y; g.h_out = h_out; g.x = x; g.stats = stats;
    g.run = edge_run_forward(plan, g.d);
    g.past = plan->T * g.d * (edge->post_gain ? edge->pre_gain ? 4 : 3 : 2) * 2 > int64_t(192) << 20;
    ProfScope prof(plan, MLORA_K_EDGE_FWD, (hipStream_t)stream);
    if (plan->dtype == MLORA_F32) launch_edge<float>(g, plan->num_cus, true, (hipStream_t)stream);
    else                          launch_edge<u16>(g, plan->num_cus, true, (hipStream_t)stream);
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}

extern "C" size_t multi_lora_edge_workspace_bytes(const mlora_plan* plan, int64_t d) {
    if (!plan || d < 1 || d > kMaxEdgeCols) return 0;
    return (size_t)edge_slots(plan, d) * (size_t)(2 * d + 1) * sizeof(float);
}

extern "C" int multi_lora_edge_bwd(mlora_plan* plan, const mlora_edge* edge, const void* h, const void* y, const float* stats, const void* dx,
                                   const void* dh_out, void* dh, void* dy, const mlora_edge_grads* grads, void* workspace, uint32_t flags,
                                   void* stream) {
    int rc = check_edge(plan, edge);
    if (rc != MLORA_OK) return rc;
    if (flags & ~MLORA_FLAG_ACCUM_GRADS) { set_error("unknown flag bits"); return MLORA_ERR_FLAGS; }
    const mlora_edge_grads none{};
    const mlora_edge_grads& G = grads ? *grads : none;
    const bool post = edge->post_gain, pre = edge->pre_gain;
    if ((!post && (G.d_post || G.d_gate || G.d_scale)) || (!pre && G.d_pre) || (!edge->gate && G.d_gate) || (!edge->res_scale && G.d_scale)) {
        set_error("block edge: the gradient of something that is not given");
        return MLORA_ERR_NULL;
    }
    if (plan->T > 0 && (!dh || !stats || (post && (!y || !dy)) || (pre && (!dx || !h)))) {
        set_error("block edge: stats, dh, y, dy, dx or h is NULL although its norm is given");
        return MLORA_ERR_NULL;
    }
    const bool wantC = G.d_post || G.d_gate, wantD = G.d_pre, wantS = G.d_scale, want = wantC || wantD || wantS;
    if (want && plan->T > 0 && !workspace) { set_error("block edge: workspace is NULL"); return MLORA_ERR_WORKSPACE; }
    if ((rc = check_element_aligned(plan, {h, y, dx, dh_out, dh, dy, edge->post_gain, edge->gate, edge->pre_gain, G.d_post, G.d_gate, G.d_pre},
                                    {stats, edge->res_scale, workspace, G.d_scale})) != MLORA_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    EdgeArgs g = edge_args(plan, edge);
    g.h = h; g.y = y; g.stats = const_cast<float*>(stats); g.dx = dx; g.dh_out = dh_out; g.dh = dh; g.dy = dy;
    g.run = edge_run(plan, g.d);
    const int64_t slots = edge_slots(plan, g.d);
    float* ws = (float*)workspace;
    if (wantC) g.partC = ws;
    if (wantD) g.partD = ws + slots * g.d;
    if (wantS) g.partS = ws + 2 * slots * g.d;
    const bool f32 = plan->dtype == MLORA_F32;
    if (plan->T > 0) {
        ProfScope prof(plan, MLORA_K_EDGE_BWD, st);
        if (f32) launch_edge<float>(g, plan->num_cus, false, st); else launch_edge<u16>(g, plan->num_cus, false, st);
    }
    if (want) {
        EdgeReduceArgs r{};
        r.d = g.d; r.N = g.N; r.run = g.run; r.off = g.off; r.post = g.post; r.post_ld = g.post_ld; r.gate = g.gate; r.gate_ld = g.gate_ld;
        r.pre_ld = g.pre_ld; r.scale = g.scale; r.partC = g.partC; r.partD = g.partD; r.partS = g.partS;
        r.d_post = G.d_post; r.d_gate = G.d_gate; r.d_pre = G.d_pre; r.d_scale = G.d_scale;
        r.accum = (flags & MLORA_FLAG_ACCUM_GRADS) ? 1 : 0;
        const unsigned tiles = (unsigned)((g.d + 63) / 64);
        ProfScope prof(plan, MLORA_K_EDGE_REDUCE, st);
        if (f32) hipLaunchKernelGGL(edge_reduce_kernel<float>, dim3(tiles, g.N), dim3(512), 0, st, r);
        else     hipLaunchKernelGGL(edge_reduce_kernel<u16>, dim3(tiles, g.N), dim3(512), 0, st, r);
        if ((G.d_post && !g.post_ld) || (G.d_gate && !g.gate_ld) || (G.d_pre && !g.pre_ld)) {
            if (f32) hipLaunchKernelGGL(edge_shared_kernel<float>, dim3(tiles), dim3(256), 0, st, r);
            else     hipLaunchKernelGGL(edge_shared_kernel<u16>, dim3(tiles), dim3(256), 0, st, r);
        }
    }
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}
