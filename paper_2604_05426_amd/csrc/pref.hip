// Preference loss (paired log ratios) from logits, and its gradient, for the pairs of many adapters in one flat token buffer.
//
//   row       m_t = max_v z_tv,  s_t = sum_v exp(z_tv - m_t),  l_t = (z_t,target - m_t) - log s_t      (rows without a target are not counted)
//   sequence  l_q = sum of its counted rows
//   pair j    m_j = beta_i ((l_c - ref_c) - (l_r - ref_r)),  c = 2 j chosen, r = 2 j + 1 rejected, i the pair's adapter
//             f_j = -(1 - a_i) log sigma(m_j) - a_i log sigma(-m_j) - u_i l_c / n_c      (n_c counted rows of c; no such term at 0)
//   adapter   loss_i = mean of f_j over its pairs
//   gradient  dz_tv = k_q(t) (1[v = target] - exp(z_tv - m_t) / s_t),  k_q = d loss / d l_q
// The rows are one stream over the vocabulary with the running maximum and sum of a softmax; everything behind it is a few numbers
// a sequence.  m_t and s_t stay apart: their one number m_t + log s_t would be rounded as its magnitude is, by 3e-5 at logits of 1000, though a row shifted
// by a constant is the same row.  From a row's sum on, log-probabilities, sequences and margins are held in 64 bits: log-probabilities of long sequences are
// large and their difference is not.
#include <cmath>
#include <cstring>
#include <new>

#include "stream_common.h"

namespace mlora {

constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = (float)(1.4426950408889634 - (double)kLog2e);

struct PrefView {
    int64_t T, V;
    int32_t N, P;
    const int32_t* seq_off;      // [2 P + 1]
    const int32_t* row_seq;      // [T]
    const int32_t* owner;        // [P]
    const int32_t* pair_start;   // [N + 1]: places of the adapters' pairs in pair_list
    const int32_t* pair_list;    // [P], by adapter, ascending
    const mlora_pref_params* params;   // [N]
    uint32_t* arrived;           // pairs done; zero between launches
};

}  // namespace mlora

struct mlora_pref {
    int dtype = 0;
    mlora::DeviceBlock block;
    mlora::PrefView view{};
};

namespace mlora {

// A row is worked on in parts of kPart columns, one work group each, whatever the batch: a row's bits do not depend on how many rows there are, and
// a few long rows have work groups for the whole chip.
// Vocabularies of up to kFewColumns take a wavefront a row, four rows a work group: 16384 rows of 512 bf16 in 32 pairs, forward (both kernels) 20 us instead
// of 42, backward 6 instead of 16; of 2048, 27 instead of 46 and 22 instead of 25.  (Up to 4096: rows of 4000, 38 instead of 52 and 41 instead of 42, but
// smaller ones up to a tenth more, by the registers.)
constexpr int kPart = 16384, kFewColumns = 2048;
// pieces of sixteen bytes of a lane, of THREADS that share a part
template <typename T, int THREADS> constexpr int kLanePieces = (THREADS == 256 ? kPart : kFewColumns) / (THREADS * kEpc<T>);
static inline int32_t pref_parts(int64_t V) { return (int32_t)((V + kPart - 1) / kPart); }

struct Softmax {       // running maximum m and sum of exp(z - m)
    float m, s;
};

// What a forward leaves for the backward, and what the kernels hand on.
struct PrefWorkspace {
    Softmax* part;       // [T][parts]
    float* target;       // [T]: logit of the row's target
    float* top;          // [T]: the row's maximum
    float* inv;          // [T]: 1 / sum of exp(z - maximum)
    float* coef;         // [2 P]
    float* pair_loss;    // [P]
};
static size_t pref_workspace_bytes(const PrefView& v) {
    return sizeof(float) * (((size_t)pref_parts(v.V) * 2 + 3) * (size_t)v.T + 3 * (size_t)v.P) + 64;
}
static PrefWorkspace pref_workspace(const PrefView& v, void* ws) {
    float* f = (float*)ws + 2 * (size_t)pref_parts(v.V) * v.T;
    return {(Softmax*)ws, f, f + v.T, f + 2 * v.T, f + 3 * v.T, f + 3 * v.T + 2 * v.P};
}

// exp(x) with both parts of log2 e: the 1.3e-8 that its fp32 value lacks would take 4e-8 off every row's log-sum in the same direction, and the margin of a pair with
// ten thousand rows more on one side is a few units.  What is left is the instruction's own, -3.4e-9 on average (measured over [-30, 0]).
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, x * kLog2eRest)); }
// maximum to subtract: a row of nothing but -inf keeps exp(-inf) = 0 instead of a NaN
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Softmax join(Softmax a, Softmax b) {
    const float m = fmaxf(a.m, b.m), f = finite_max(m);
    return {m, a.s * exp_of(a.m - f) + b.s * exp_of(b.m - f)};
}

__device__ __forceinline__ bool counted_target(const PrefView& g, int32_t target) { return target >= 0 && target < g.V; }

// Elements inside the row of a lane's piece u, which starts at column c0 + u * THREADS * kEpc.
template <typename T, int THREADS> __device__ __forceinline__ int part_valid(const PrefView& g, int64_t c0, int u) {
    return (int)max((int64_t)0, min((int64_t)kEpc<T>, g.V - c0 - u * THREADS * kEpc<T>));
}

// Maximum and sum of a lane's elements of one part.  All of them are on their way at a time; the maximum is taken before the sum, so that no sum is scaled
// again.  FULL: the part does not pass the end of the row.
template <typename T, bool FULL, int THREADS> __device__ __forceinline__ Softmax lane_softmax(const PrefView& g, const T* row, int64_t c0) {
    uint4 p[kLanePieces<T, THREADS>];
    auto valid_of = [&](int u) { return FULL ? kEpc<T> : part_valid<T, THREADS>(g, c0, u); };
#pragma unroll
    for (int u = 0; u < kLanePieces<T, THREADS>; ++u) {
        const int valid = valid_of(u);
        if (valid > 0) p[u] = load16(row + c0 + u * THREADS * kEpc<T>, valid);
    }
    Softmax a = {-INFINITY, 0.f};
#pragma unroll
    for (int u = 0; u < kLanePieces<T, THREADS>; ++u) {
        const int valid = valid_of(u);
        if (valid <= 0) continue;
        float x[kEpc<T>];
        unpack16<T>(p[u], x);
#pragma unroll
        for (int k = 0; k < kEpc<T>; ++k) a.m = fmaxf(a.m, k < valid ? x[k] : -INFINITY);
    }
    const float f = finite_max(a.m);
#pragma unroll
    for (int u = 0; u < kLanePieces<T, THREADS>; ++u) {
        const int valid = valid_of(u);
        if (valid <= 0) continue;
        float x[kEpc<T>];
        unpack16<T>(p[u], x);
#pragma unroll
        for (int k = 0; k < kEpc<T>; ++k) a.s += k < valid ? exp_of(x[k] - f) : 0.f;
    }
    return a;
}

__device__ __forceinline__ Softmax wave_join(Softmax a) {
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) a = join(a, Softmax{__shfl_xor(a.m, w), __shfl_xor(a.s, w)});
    return a;
}

// Maximum and sum of one part of one row.  A stream: 4096 x 128256 bf16, seven tenths of the rows counted (735 MB), 130 - 150 us.
template <typename T>
__global__ __launch_bounds__(256) void pref_rows_kernel(PrefView g, const T* z, int64_t ld, const int32_t* targets, PrefWorkspace ws, int32_t parts) {
    const int64_t t = blockIdx.x / (uint32_t)parts;
    const int part = (int)(blockIdx.x - (uint32_t)t * (uint32_t)parts);
    const int32_t target = targets[t];
    if (!counted_target(g, target)) return;
    const T* row = z + t * ld;
    const int64_t c0 = (int64_t)part * kPart + threadIdx.x * kEpc<T>;
    Softmax a = (part + 1) * (int64_t)kPart <= g.V ? lane_softmax<T, true, 256>(g, row, c0) : lane_softmax<T, false, 256>(g, row, c0);
    a = wave_join(a);
    __shared__ Softmax wave[4];
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = a;
    __syncthreads();
    if (threadIdx.x == 0) {
        ws.part[(int64_t)t * parts + part] = join(join(wave[0], wave[1]), join(wave[2], wave[3]));
        if (target / kPart == part) ws.target[t] = to_f32<T>(row[target]);
    }
}
template <typename T>
__global__ __launch_bounds__(256) void pref_few_rows_kernel(PrefView g, const T* z, int64_t ld, const int32_t* targets, PrefWorkspace ws) {
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= g.T) return;
    const int32_t target = targets[t];
    if (!counted_target(g, target)) return;
    const int lane = threadIdx.x & 63;
    const T* row = z + t * ld;
    const Softmax a = wave_join(lane_softmax<T, false, 64>(g, row, lane * kEpc<T>));
    if (lane == 0) {
        ws.part[t] = a;
        ws.target[t] = to_f32<T>(row[target]);
    }
}

// Log-probability of a counted row from its parts, in their order; its maximum and the sum's inverse.
__device__ __forceinline__ double row_result(const PrefWorkspace& ws, int64_t t, int32_t parts, float& top, float& inv) {
    const Softmax* p = ws.part + t * parts;
    float m = -INFINITY;
    double s = 0.0;
    for (int k = 0; k < parts; k += 8) {        // eight on their way at a time
        Softmax b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = k + j < parts ? p[k + j] : Softmax{-INFINITY, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float to = fmaxf(m, b[j].m), f = finite_max(to);
            s = s * (double)exp_of(m - f) + (double)b[j].s * (double)exp_of(b[j].m - f);
            m = to;
        }
    }
    top = finite_max(m);
    inv = (float)(1.0 / s);
    return ((double)ws.target[t] - (double)top) - log(s);
}

// Sum of a sequence's rows by 256 threads (`tid` of them), and how many of them are counted; red and cnt hold a number per wavefront.  The caller puts a
// barrier behind.
__device__ __forceinline__ void sequence_sum(const PrefView& g, const PrefWorkspace& ws, const int32_t* targets, int32_t parts, int q, int tid, float* row_out,
                                             double* red, int32_t* cnt) {
    double l = 0.0;
    int n = 0;
    const int64_t end = g.seq_off[q + 1];
    for (int64_t t = g.seq_off[q] + tid; t < end; t += 256) {
        float top, inv;
        double v = row_result(ws, t, parts, top, inv);      // (of any row, so that its loads do not wait for the target)
        if (counted_target(g, targets[t])) {
            ws.top[t] = top;
            ws.inv[t] = inv;
            l += v;
            ++n;
        } else {
            v = 0.0;
        }
        if (row_out) row_out[t] = (float)v;
    }
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) { l += __shfl_xor(l, w); n += __shfl_xor(n, w); }
    if ((tid & 63) == 0) { red[tid >> 6] = l; cnt[tid >> 6] = n; }
}

// The sequences' log-probabilities alone; one work group per sequence.
__global__ __launch_bounds__(256) void pref_sums_kernel(PrefView g, const int32_t* targets, PrefWorkspace ws, int32_t parts, float* row_out, float* logp) {
    __shared__ double red[4];
    __shared__ int32_t cnt[4];
    sequence_sum(g, ws, targets, parts, blockIdx.x, threadIdx.x, row_out, red, cnt);
    __syncthreads();
    if (threadIdx.x == 0) logp[blockIdx.x] = (float)((red[0] + red[1]) + (red[2] + red[3]));
}

// One work group per pair, half of it for each sequence; the last one to finish takes the adapters' means, in the order of the pairs.
__global__ __launch_bounds__(512) void pref_pairs_kernel(PrefView g, const int32_t* targets, const float* ref, PrefWorkspace ws, int32_t parts, float* logp,
                                                         float* margin, float* loss) {
    __shared__ double red[8];
    __shared__ int32_t cnt[8];
    __shared__ bool last;
    const int j = blockIdx.x, half = threadIdx.x >> 8;
    const int i = g.owner[j];
    const mlora_pref_params prm = g.params[i];
    const int pairs = g.pair_start[i + 1] - g.pair_start[i];
    const float refs[2] = {ref ? ref[2 * j] : 0.f, ref ? ref[2 * j + 1] : 0.f};
    sequence_sum(g, ws, targets, parts, 2 * j + half, threadIdx.x & 255, nullptr, red + 4 * half, cnt + 4 * half);
    __syncthreads();
    if (threadIdx.x == 0) {
        const double lc = (red[0] + red[1]) + (red[2] + red[3]), lr = (red[4] + red[5]) + (red[6] + red[7]);
        const int nc = (cnt[0] + cnt[1]) + (cnt[2] + cnt[3]);
        const double rc = (double)refs[0], rr = (double)refs[1];
        const double m = (double)prm.beta * ((lc - rc) - (lr - rr)), a = (double)prm.label_smoothing;
        const double e = exp(-fabs(m)), soft = log1p(e);
        const double lo = fmax(-m, 0.0) + soft, hi = fmax(m, 0.0) + soft;      // -log sigma(m), -log sigma(-m)
        // a term without weight has no part where its factor is infinite (a sequence of probability 0)
        double f = 0.0;
        if (a < 1.0) f += (1.0 - a) * lo;
        if (a > 0.0) f += a * hi;
        const double w = nc > 0 ? (double)prm.nll_weight / nc : 0.0;
        if (w != 0.0) f -= w * lc;
        const double near = 1.0 / (1.0 + e), far = e * near;                 // sigma(|m|), sigma(-|m|)
        const double dm = (double)prm.beta * (a * (m >= 0.0 ? near : far) - (1.0 - a) * (m >= 0.0 ? far : near));
        const double share = 1.0 / pairs;
        ws.coef[2 * j] = (float)(share * (dm - w));
        ws.coef[2 * j + 1] = (float)(-share * dm);
        logp[2 * j] = (float)lc;
        logp[2 * j + 1] = (float)lr;
        if (margin) margin[j] = (float)m;
        __hip_atomic_store(&ws.pair_loss[j], (float)f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(g.arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1u == (uint32_t)g.P;
    }
    __syncthreads();
    if (!last) return;
    for (int i = threadIdx.x; i < g.N; i += 512) {
        double s = 0.0;
        const int a = g.pair_start[i], b = g.pair_start[i + 1];
        for (int k = a; k < b; ++k) s += (double)__hip_atomic_load(&ws.pair_loss[g.pair_list[k]], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        loss[i] = b > a ? (float)(s / (b - a)) : 0.f;
    }
    if (threadIdx.x == 0) __hip_atomic_store(g.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__global__ void pref_no_pairs_kernel(int32_t N, float* loss) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < N) loss[i] = 0.f;
}

// Gradient of a lane's elements of one part.  Each lane reads its elements before it writes them, and a piece that passes the end of its row is read element
// by element: dz may be z.
template <typename T, bool FULL, int THREADS>
__device__ __forceinline__ void lane_gradient(const PrefView& g, const T* row, T* out, int64_t c0, int64_t target, float k, float top, float inv) {
    uint4 p[kLanePieces<T, THREADS>];
    auto valid_of = [&](int u) { return FULL ? kEpc<T> : part_valid<T, THREADS>(g, c0, u); };
#pragma unroll
    for (int u = 0; u < kLanePieces<T, THREADS>; ++u) {
        const int valid = valid_of(u);
        if (valid > 0) p[u] = load16(row + c0 + u * THREADS * kEpc<T>, valid);
    }
    const int64_t hit = target - c0;
#pragma unroll
    for (int u = 0; u < kLanePieces<T, THREADS>; ++u) {
        const int valid = valid_of(u);
        if (valid <= 0) continue;
        float x[kEpc<T>];
        unpack16<T>(p[u], x);
#pragma unroll
        for (int e = 0; e < kEpc<T>; ++e) {
            const float pr = exp_of(x[e] - top) * inv;
            x[e] = k * ((hit == u * THREADS * kEpc<T> + e ? 1.f : 0.f) - pr);
        }
        store16(out + c0 + u * THREADS * kEpc<T>, pack16<T>(x), valid);
    }
}

// Gradient of the part of row t whose first column for this lane is c0; full: it does not pass the end of the row.
template <typename T, int THREADS>
__device__ __forceinline__ void row_gradient(const PrefView& g, const T* z, int64_t ld, const int32_t* targets, const float* dloss, const PrefWorkspace& ws, T* dz,
                                             int64_t ldd, int64_t t, int64_t c0, bool full) {
    const int32_t target = targets[t];
    T* out = dz + t * ldd;
    if (!counted_target(g, target)) {
#pragma unroll
        for (int u = 0; u < kLanePieces<T, THREADS>; ++u) {
            const int valid = part_valid<T, THREADS>(g, c0, u);
            if (valid > 0) store16(out + c0 + u * THREADS * kEpc<T>, zero4(), valid);
        }
        return;
    }
    const T* row = z + t * ld;
    const int q = g.row_seq[t];
    const float k = ws.coef[q] * (dloss ? dloss[g.owner[q >> 1]] : 1.f), top = ws.top[t], inv = ws.inv[t];
    if (full) lane_gradient<T, true, THREADS>(g, row, out, c0, target, k, top, inv);
    else      lane_gradient<T, false, THREADS>(g, row, out, c0, target, k, top, inv);
}

// Gradient of one part of one row (the same: 735 MB in, 1051 out, 305 us, 5.9 TB/s), the last rows first: the forward read them last, and what the caches still hold of the logits is theirs.
template <typename T>
__global__ __launch_bounds__(256) void pref_grad_kernel(PrefView g, const T* z, int64_t ld, const int32_t* targets, const float* dloss, PrefWorkspace ws,
                                                        T* dz, int64_t ldd, int32_t parts) {
    const uint32_t block = gridDim.x - 1 - blockIdx.x;
    const int64_t t = block / (uint32_t)parts;
    const int part = (int)(block - (uint32_t)t * (uint32_t)parts);
    row_gradient<T, 256>(g, z, ld, targets, dloss, ws, dz, ldd, t, (int64_t)part * kPart + threadIdx.x * kEpc<T>, (part + 1) * (int64_t)kPart <= g.V);
}
template <typename T>
__global__ __launch_bounds__(256) void pref_few_grad_kernel(PrefView g, const T* z, int64_t ld, const int32_t* targets, const float* dloss, PrefWorkspace ws,
                                                            T* dz, int64_t ldd) {
    const int64_t t = (int64_t)(gridDim.x - 1 - blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (t < g.T) row_gradient<T, 64>(g, z, ld, targets, dloss, ws, dz, ldd, t, (threadIdx.x & 63) * kEpc<T>, false);
}

static int check_rows(const mlora_pref* p, const void* z, int64_t ld, const void* targets, const void* ws) {
    if (!p) { set_error("pref is NULL"); return MLORA_ERR_NULL; }
    if (ld < p->view.V) { set_error("preference loss: a row stride below the vocabulary"); return MLORA_ERR_SHAPE; }
    if (p->view.T == 0 && p->view.P == 0) return MLORA_OK;
    if (p->view.T > 0 && (!z || !targets)) { set_error("logits / targets is NULL"); return MLORA_ERR_NULL; }
    if (!ws) { set_error("workspace is NULL"); return MLORA_ERR_WORKSPACE; }
    if (((uintptr_t)z & (p->dtype == MLORA_F32 ? 3 : 1)) || (((uintptr_t)targets | (uintptr_t)ws) & 3)) {
        set_error("preference loss: a tensor is not aligned to its elements");
        return MLORA_ERR_ALIGN;
    }
    return MLORA_OK;
}

static void launch_rows(const mlora_pref* p, const void* z, int64_t ld, const int32_t* targets, const PrefWorkspace& ws, hipStream_t st) {
    const PrefView& v = p->view;
    if (v.T == 0) return;
    const bool f32 = p->dtype == MLORA_F32;
    if (v.V <= kFewColumns) {
        const dim3 grid((unsigned)((v.T + 3) / 4));
        if (f32) hipLaunchKernelGGL(pref_few_rows_kernel<float>, grid, dim3(256), 0, st, v, (const float*)z, ld, targets, ws);
        else     hipLaunchKernelGGL(pref_few_rows_kernel<u16>, grid, dim3(256), 0, st, v, (const u16*)z, ld, targets, ws);
        return;
    }
    const int32_t parts = pref_parts(v.V);
    const dim3 grid((unsigned)(v.T * parts));
    if (f32) hipLaunchKernelGGL(pref_rows_kernel<float>, grid, dim3(256), 0, st, v, (const float*)z, ld, targets, ws, parts);
    else     hipLaunchKernelGGL(pref_rows_kernel<u16>, grid, dim3(256), 0, st, v, (const u16*)z, ld, targets, ws, parts);
}

}  // namespace mlora

using namespace mlora;

extern "C" int multi_lora_pref_create(mlora_pref** out, int dtype, int64_t T, int64_t V, int32_t N, int32_t n_pairs, const int32_t* pair_adapter,
                                      const int64_t* seq_offsets, const mlora_pref_params* params, void* stream) {
    if (!out) { set_error("out is NULL"); return MLORA_ERR_NULL; }
    *out = nullptr;
    if (dtype != MLORA_F32 && dtype != MLORA_BF16) { set_error("dtype must be MLORA_F32 or MLORA_BF16"); return MLORA_ERR_DTYPE; }
    if (T < 0 || T > INT32_MAX || V < 1 || V > INT32_MAX || N < 1 || N > MLORA_MAX_ADAPTERS || n_pairs < 0 || n_pairs > (1 << 22)) {
        set_error("preference loss: T, V, N or n_pairs out of range");
        return MLORA_ERR_SHAPE;
    }
    if (T * pref_parts(V) >= 1 << 24) {      // work groups of 256 threads; a launch has fewer than 2^32
        set_error("preference loss: 2^24 or more parts of 16384 columns in T rows");
        return MLORA_ERR_SHAPE;
    }
    if (!params || !seq_offsets || (n_pairs > 0 && !pair_adapter)) { set_error("params / seq_offsets / pair_adapter is NULL"); return MLORA_ERR_NULL; }
    const int32_t S = 2 * n_pairs;
    if (seq_offsets[0] != 0 || seq_offsets[S] != T) { set_error("sequence offsets do not start at 0 or do not end at T"); return MLORA_ERR_SEGMENTS; }
    for (int32_t q = 0; q < S; ++q)
        if (seq_offsets[q + 1] < seq_offsets[q]) { set_error("sequence offsets decrease"); return MLORA_ERR_SEGMENTS; }
    for (int32_t j = 0; j < n_pairs; ++j)
        if (pair_adapter[j] < 0 || pair_adapter[j] >= N) { set_error("a pair's adapter is outside [0, N)"); return MLORA_ERR_SEGMENTS; }
    for (int32_t i = 0; i < N; ++i)
        if (!std::isfinite(params[i].beta) || !(params[i].label_smoothing >= 0.f && params[i].label_smoothing <= 1.f) || !std::isfinite(params[i].nll_weight)) {
            set_error("preference loss: beta or nll_weight is not finite, or label_smoothing is outside [0, 1]");
            return MLORA_ERR_SCALE;
        }
    try {
        std::unique_ptr<mlora_pref> p(new mlora_pref);
        p->dtype = dtype;
        auto up = [](size_t b) { return (b + 255) & ~size_t(255); };
        const size_t o_off = 256, o_row = o_off + up(4 * ((size_t)S + 1)), o_own = o_row + up(4 * (size_t)T), o_start = o_own + up(4 * (size_t)n_pairs),
                     o_list = o_start + up(4 * ((size_t)N + 1)), o_prm = o_list + up(4 * (size_t)n_pairs), total = o_prm + up(sizeof(mlora_pref_params) * (size_t)N);
        std::vector<unsigned char> host(total, 0);
        int32_t* h_off = (int32_t*)(host.data() + o_off); int32_t* h_row = (int32_t*)(host.data() + o_row);
        int32_t* h_start = (int32_t*)(host.data() + o_start); int32_t* h_list = (int32_t*)(host.data() + o_list);
        for (int32_t q = 0; q <= S; ++q) h_off[q] = (int32_t)seq_offsets[q];
        for (int32_t q = 0; q < S; ++q)
            for (int64_t t = seq_offsets[q]; t < seq_offsets[q + 1]; ++t) h_row[t] = q;
        if (n_pairs) std::memcpy(host.data() + o_own, pair_adapter, 4 * (size_t)n_pairs);
        for (int32_t j = 0; j < n_pairs; ++j) ++h_start[pair_adapter[j] + 1];
        for (int32_t i = 0; i < N; ++i) h_start[i + 1] += h_start[i];
        std::vector<int32_t> at(h_start, h_start + N);
        for (int32_t j = 0; j < n_pairs; ++j) h_list[at[pair_adapter[j]]++] = j;
        std::memcpy(host.data() + o_prm, params, sizeof(mlora_pref_params) * (size_t)N);
        MLORA_HIP_TRY(hipMalloc(&p->block.ptr, total));
        unsigned char* d = (unsigned char*)p->block.ptr;
        hipStream_t st = (hipStream_t)stream;
        MLORA_HIP_TRY(hipMemcpyAsync(d, host.data(), total, hipMemcpyHostToDevice, st));
        MLORA_HIP_TRY(hipStreamSynchronize(st));
        p->view = {T, V, N, n_pairs, (const int32_t*)(d + o_off), (const int32_t*)(d + o_row), (const int32_t*)(d + o_own), (const int32_t*)(d + o_start),
                   (const int32_t*)(d + o_list), (const mlora_pref_params*)(d + o_prm), (uint32_t*)d};
        *out = p.release();
    } catch (const std::bad_alloc&) {
        set_error("out of host memory");
        return MLORA_ERR_SHAPE;
    }
    return MLORA_OK;
}

extern "C" int multi_lora_pref_destroy(mlora_pref* pref) {
    delete pref;
    return MLORA_OK;
}

extern "C" size_t multi_lora_pref_workspace_bytes(const mlora_pref* pref) { return pref ? pref_workspace_bytes(pref->view) : 0; }

extern "C" int multi_lora_pref_logp(mlora_pref* pref, const void* logits, int64_t ld, const int32_t* targets, float* row_logp, float* logp, void* workspace,
                                    void* stream) {
    int rc = check_rows(pref, logits, ld, targets, workspace);
    if (rc != MLORA_OK) return rc;
    const PrefView& v = pref->view;
    if (v.P > 0 && !logp) { set_error("logp is NULL"); return MLORA_ERR_NULL; }
    if (((uintptr_t)row_logp | (uintptr_t)logp) & 3) { set_error("row_logp / logp is not 4-byte aligned"); return MLORA_ERR_ALIGN; }
    hipStream_t st = (hipStream_t)stream;
    const PrefWorkspace ws = pref_workspace(v, workspace);
    launch_rows(pref, logits, ld, targets, ws, st);
    if (v.P > 0) hipLaunchKernelGGL(pref_sums_kernel, dim3((unsigned)(2 * v.P)), dim3(256), 0, st, v, targets, ws, pref_parts(v.V), row_logp, logp);
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}

extern "C" int multi_lora_pref_fwd(mlora_pref* pref, const void* logits, int64_t ld, const int32_t* targets, const float* ref_logp, float* logp, float* margin,
                                   float* loss, void* workspace, void* stream) {
    int rc = check_rows(pref, logits, ld, targets, workspace);
    if (rc != MLORA_OK) return rc;
    const PrefView& v = pref->view;
    if (!loss || (v.P > 0 && !logp)) { set_error("logp / loss is NULL"); return MLORA_ERR_NULL; }
    if (((uintptr_t)ref_logp | (uintptr_t)logp | (uintptr_t)margin | (uintptr_t)loss) & 3) {
        set_error("ref_logp / logp / margin / loss is not 4-byte aligned");
        return MLORA_ERR_ALIGN;
    }
    hipStream_t st = (hipStream_t)stream;
    const PrefWorkspace ws = pref_workspace(v, workspace);
    launch_rows(pref, logits, ld, targets, ws, st);
    if (v.P > 0) hipLaunchKernelGGL(pref_pairs_kernel, dim3((unsigned)v.P), dim3(512), 0, st, v, targets, ref_logp, ws, pref_parts(v.V), logp, margin, loss);
    else         hipLaunchKernelGGL(pref_no_pairs_kernel, dim3((unsigned)(v.N + 255) / 256), dim3(256), 0, st, v.N, loss);
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}

extern "C" int multi_lora_pref_bwd(mlora_pref* pref, const void* logits, int64_t ld, const int32_t* targets, const float* dloss, void* dlogits, int64_t ldd,
                                   const void* workspace, void* stream) {
    int rc = check_rows(pref, logits, ld, targets, workspace);
    if (rc != MLORA_OK) return rc;
    const PrefView& v = pref->view;
    if (ldd < v.V) { set_error("preference loss: a row stride below the vocabulary"); return MLORA_ERR_SHAPE; }
    if (v.T == 0) return MLORA_OK;
    if (!dlogits) { set_error("dlogits is NULL"); return MLORA_ERR_NULL; }
    if (dlogits == logits && ldd != ld && v.T > 1) {      // rows would be written before others' have been read
        set_error("preference loss: in place with another row stride");
        return MLORA_ERR_SHAPE;
    }
    if (((uintptr_t)dlogits & (pref->dtype == MLORA_F32 ? 3 : 1)) || ((uintptr_t)dloss & 3)) {
        set_error("dlogits / dloss is not aligned to its elements");
        return MLORA_ERR_ALIGN;
    }
    hipStream_t st = (hipStream_t)stream;
    const PrefWorkspace ws = pref_workspace(v, const_cast<void*>(workspace));
    const bool f32 = pref->dtype == MLORA_F32;
    const float* const zf = (const float*)logits;
    const u16* const zh = (const u16*)logits;
    if (v.V <= kFewColumns) {
        const dim3 grid((unsigned)((v.T + 3) / 4));
        if (f32) hipLaunchKernelGGL(pref_few_grad_kernel<float>, grid, dim3(256), 0, st, v, zf, ld, targets, dloss, ws, (float*)dlogits, ldd);
        else     hipLaunchKernelGGL(pref_few_grad_kernel<u16>, grid, dim3(256), 0, st, v, zh, ld, targets, dloss, ws, (u16*)dlogits, ldd);
    } else {
        const int32_t parts = pref_parts(v.V);
        const dim3 grid((unsigned)(v.T * parts));
        if (f32) hipLaunchKernelGGL(pref_grad_kernel<float>, grid, dim3(256), 0, st, v, zf, ld, targets, dloss, ws, (float*)dlogits, ldd, parts);
        else     hipLaunchKernelGGL(pref_grad_kernel<u16>, grid, dim3(256), 0, st, v, zh, ld, targets, dloss, ws, (u16*)dlogits, ldd, parts);
    }
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}
