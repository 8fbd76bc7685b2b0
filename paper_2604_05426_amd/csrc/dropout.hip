// Dropout of the LoRA branch: every adapter has its own rate and key, the mask comes from a counter-based generator and is never
// stored.
//
// Ten rounds of the Philox 4 x 32 bijection (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011)
// turn the counter (column / 8, row in the segment, 64-bit counter) into 128 bits under the adapter's 64-bit key: eight 16-bit
// numbers, one for each of eight consecutive columns.  An element is kept where its number is not below round(65536 p), so the rate is
// p to within 2^-17, and a kept one is divided by the share that is really kept.  The row counts from the start of the segment: a
// job's mask does not depend on who shares its batch.  A dropped element is a zero by selection, not by a product, so Inf and NaN
// do not get through the mask.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "stream_common.h"

namespace mlora {

struct DropEntry {
    int32_t row0, rows;        // the adapter's segment
    int32_t end;               // row blocks up to the end of this adapter
    uint32_t threshold;        // 0 .. 65536
    float inv;                 // 65536 / (65536 - threshold), 0 where nothing is kept
    uint32_t key0, key1;
    int32_t pad;
};
constexpr int kDropBatch = 64, kDropFew = 8;
constexpr int64_t kMaxDropCols = int64_t(65535) * 256 * 4;      // blockIdx.y counts groups of up to 256 lanes' columns
struct DropCall {
    const void* X; int64_t ldx;
    const void* add; int64_t ldadd;
    void* Y; int64_t ldy;
    int64_t cols;
    const uint64_t* step;
    uint64_t counter;
    int32_t count, log_tpr;    // 2^log_tpr threads side by side on a row
    int32_t base;              // row blocks before this launch
};
// A launch's adapters travel in its arguments, room for eight or for 64: two kilobytes of arguments cost a launch more than a small call's kernel can win
// (256 x 256, four adapters: 4.6 / 5.0 us a call).
template <int N> struct DropArgs : DropCall {
    DropEntry e[N];
};
static_assert(sizeof(DropArgs<kDropBatch>) <= 4096, "");

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
        c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
        c[3] = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// A work group takes 256 / tpr rows at a time, kDropRows times; blockIdx.y names the group of tpr lanes' columns.  A lane takes sixteen bytes of a row: the
// eight columns of a counter, or half of them in fp32, where two lanes run the generator on the same counter (lines loaded and stored in halves
// cost more: 4096 x 8192 with addend 84.7 us, whole 77).  Bound by memory: with one round of the generator instead of ten it takes the
// same time.  More rows a lane do not help (kDropRows 8, 4, 2: 154, 149, 144 us for 32686 x 4096 with addend).
// PAST: tensors that do not fit three quarters of the Infinity Cache together go past the caches (144 -> 127 us, 6.3 TB/s; 16384 x 4096 without addend 50 -> 45); smaller ones stay
// there for whoever reads them next (4096 x 4096 itself takes 13.3 and, past the caches, 14.3 us).
constexpr int kDropRows = 2;
template <typename T, bool ADD, bool PAST, int N>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs<N> g) {
    constexpr int E = kEpc<T>, U = kDropRows;
    const int32_t wg = g.base + (int32_t)blockIdx.x;
    int32_t lo = 0, hi = g.count;            // the first adapter that ends behind this row block
    while (lo < hi) {
        const int32_t mid = (lo + hi) >> 1;
        if (g.e[mid].end <= wg) lo = mid + 1; else hi = mid;
    }
    const DropEntry& e = g.e[lo];
    const int log_tpr = g.log_tpr, side = 256 >> log_tpr;
    const int64_t col = ((int64_t)blockIdx.y * (1 << log_tpr) + (threadIdx.x & ((1 << log_tpr) - 1))) * E;
    if (col >= g.cols) return;
    const int valid = (int)min((int64_t)E, g.cols - col);
    const bool whole = g.cols >= E;
    const int32_t first = (wg - (lo > 0 ? g.e[lo - 1].end : 0)) * (side * U) + (threadIdx.x >> log_tpr);
    const uint32_t threshold = e.threshold;
    const float inv = e.inv;
    const uint64_t counter = g.counter + (g.step ? *g.step : 0);
    uint4 x[U], a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t row = first + u * side;
        if (row >= e.rows) break;
        const int64_t t = (int64_t)e.row0 + row;
        x[u] = load16_row<T, PAST>((const T*)g.X + t * g.ldx + col, valid, whole);
        if (ADD) a[u] = load16_row<T, PAST>((const T*)g.add + t * g.ldadd + col, valid, whole);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t row = first + u * side;
        if (row >= e.rows) break;
        const int64_t t = (int64_t)e.row0 + row;
        uint32_t c[4] = {(uint32_t)(col / 8), (uint32_t)row, (uint32_t)counter, (uint32_t)(counter >> 32)};
        if (threshold) philox(c, e.key0, e.key1);
        if (E == 4 && (col & 4)) { c[0] = c[2]; c[1] = c[3]; }      // the second half's numbers
        float v[E], b[E];
        unpack16<T>(x[u], v);
        if (ADD) unpack16<T>(a[u], b);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const uint32_t number = (j & 1) ? c[j >> 1] >> 16 : c[j >> 1] & 0xffffu;
            const float kept = threshold == 0 || number >= threshold ? v[j] * inv : 0.f;
            v[j] = ADD ? kept + b[j] : kept;
        }
        store16<T, PAST>((T*)g.Y + t * g.ldy + col, pack16<T>(v), valid);
    }
}

template <typename T, bool ADD> static void launch_dropout(const DropCall& call, const DropEntry* e, dim3 grid, bool past, hipStream_t st) {
    auto args = [&](auto size) {
        DropArgs<decltype(size)::value> g;
        static_cast<DropCall&>(g) = call;
        std::memcpy(g.e, e, sizeof(DropEntry) * (size_t)call.count);
        return g;
    };
    const std::integral_constant<int, kDropFew> few;
    const std::integral_constant<int, kDropBatch> many;
    if (past)                        hipLaunchKernelGGL((dropout_kernel<T, ADD, true, kDropBatch>), grid, dim3(256), 0, st, args(many));
    else if (call.count <= kDropFew) hipLaunchKernelGGL((dropout_kernel<T, ADD, false, kDropFew>), grid, dim3(256), 0, st, args(few));
    else                             hipLaunchKernelGGL((dropout_kernel<T, ADD, false, kDropBatch>), grid, dim3(256), 0, st, args(many));
}

}  // namespace mlora

using namespace mlora;

extern "C" int multi_lora_dropout(mlora_plan* plan, const mlora_dropout* drop, int64_t cols, const void* X, int64_t ldx, const void* add,
                                  int64_t ldadd, void* Y, int64_t ldy, uint64_t counter, const uint64_t* step, void* stream) {
    if (!plan || !drop) { set_error("plan / drop is NULL"); return MLORA_ERR_NULL; }
    mlora_plan* p = plan;
    if (p->N == 0) { set_error("dropout: the plan has no adapters"); return MLORA_ERR_SHAPE; }
    if (cols < 1 || cols > kMaxDropCols || ldx < cols || ldy < cols || (add && ldadd < cols)) {
        set_error("dropout: cols out of range, or a row stride below it");
        return MLORA_ERR_SHAPE;
    }
    for (int32_t i = 0; i < p->N; ++i)
        if (!(drop[i].p >= 0.f && drop[i].p <= 1.f)) { set_error("dropout: a rate is outside [0, 1]"); return MLORA_ERR_SCALE; }
    if (p->T == 0) return MLORA_OK;
    if (!X || !Y) { set_error("X / Y is NULL"); return MLORA_ERR_NULL; }
    if (p->T > 1 && ((Y == X && ldy != ldx) || (Y == add && ldy != ldadd))) {      // rows would be written before others' have been read
        set_error("dropout: in place with another row stride");
        return MLORA_ERR_SHAPE;
    }
    const uintptr_t es = p->dtype == MLORA_F32 ? 4 : 2;
    if (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)add) & (es - 1)) { set_error("X / add / Y is not aligned to its elements"); return MLORA_ERR_ALIGN; }
    if ((uintptr_t)step & 7) { set_error("step is not 8-byte aligned"); return MLORA_ERR_ALIGN; }
    hipStream_t st = (hipStream_t)stream;
    const bool f32 = p->dtype == MLORA_F32;
    const int64_t lane = f32 ? 4 : 8, pieces = (cols + lane - 1) / lane;       // sixteen bytes
    const bool past = (add ? 3 : 2) * p->T * cols * (int64_t)es > int64_t(192) << 20;
    DropCall g{};
    DropEntry entries[kDropBatch];
    g.X = X; g.ldx = ldx; g.add = add; g.ldadd = ldadd; g.Y = Y; g.ldy = ldy; g.cols = cols; g.step = step; g.counter = counter;
    while (g.log_tpr < 8 && (int64_t(1) << g.log_tpr) < pieces) ++g.log_tpr;
    const int64_t side = 256 >> g.log_tpr, groups = (pieces + (1 << g.log_tpr) - 1) >> g.log_tpr;
    for (int32_t base = 0; base < p->N;) {
        g.count = 0;
        int64_t blocks = 0;
        for (; base < p->N && g.count < kDropBatch; ++base) {
            const int64_t rows = p->off[base + 1] - p->off[base];
            if (rows == 0) continue;
            blocks += (rows + kDropRows * side - 1) / (kDropRows * side);
            DropEntry& e = entries[g.count++];
            const int32_t t = (int32_t)std::nearbyint(65536.0 * (double)drop[base].p);
            e.pad = 0;
            e.row0 = (int32_t)p->off[base]; e.rows = (int32_t)rows; e.end = (int32_t)blocks;
            e.threshold = (uint32_t)t;
            e.inv = t < 65536 ? (float)(65536.0 / (double)(65536 - t)) : 0.f;
            e.key0 = (uint32_t)drop[base].seed; e.key1 = (uint32_t)(drop[base].seed >> 32);
        }
        if (g.count == 0) break;
        ProfScope prof(p, MLORA_K_DROPOUT, st);
        for (int64_t first = 0; first < blocks; first += kMaxLaunchGroups) {
            g.base = (int32_t)first;
            const dim3 grid((unsigned)std::min(kMaxLaunchGroups, blocks - first), (unsigned)groups);
            if (f32 && add) launch_dropout<float, true>(g, entries, grid, past, st);
            else if (f32)   launch_dropout<float, false>(g, entries, grid, past, st);
            else if (add)   launch_dropout<u16, true>(g, entries, grid, past, st);
            else            launch_dropout<u16, false>(g, entries, grid, past, st);
        }
    }
    MLORA_HIP_TRY(hipGetLastError());
    return MLORA_OK;
}
