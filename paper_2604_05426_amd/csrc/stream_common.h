// Device helpers of the streaming operators (dropout, block edges, preference loss): pieces of eight elements of a row that may
// start at any element, and sums over wavefronts.
#pragma once

#include "general_common.h"

namespace mlora {

constexpr int64_t kMaxLaunchGroups = int64_t(1) << 23;      // work groups of 256 along a launch's x: a dimension holds fewer than 2^32 work items

constexpr int kPiece = 8;      // elements a lane takes at a time: 16 bytes of bf16, 32 of fp32

// Eight elements as they lie in memory.
template <typename T> struct Piece {
    uint4 w[sizeof(T) / 2];
};
template <typename T> __device__ __forceinline__ Piece<T> load_piece(const T* p) {
    Piece<T> v;
    __builtin_memcpy(&v, p, sizeof(v));
    return v;
}
// The first `valid` (one at least) elements of the piece at p, the others zero; nothing outside its row is read.  `whole` (uniform): the row holds eight
// elements or more, so that a piece that passes its end can be had as the row's last eight elements: one load, and none of the registers
// that eight separate elements in flight take (they more than doubled those of the block edges' kernels).  Loads that are to stay in flight take the two
// parts, load_raw and, where the elements are used, settle, which shifts them: a shift behind the load would wait for it (20000 x 2697 bf16 through
// a block edge's backward, all gradients: 316 instead of 203 us).
template <typename T> __device__ __forceinline__ Piece<T> load_raw(const T* p, int valid, bool whole) {
    if (whole) return load_piece(p - max(0, kPiece - valid));
    Piece<T> v;
    uint32_t w[sizeof(v) / 4];
#pragma unroll
    for (int k = 0; k < (int)sizeof(v) / 4; ++k) w[k] = 0u;
#pragma unroll 1
    for (int e = 0; e < valid; ++e) {
        uint32_t x;
        if constexpr (sizeof(T) == 4) x = __float_as_uint(p[e]);
        else x = (uint32_t)p[e] << (16 * (e & 1));
        const int at = sizeof(T) == 4 ? e : e >> 1;
#pragma unroll
        for (int k = 0; k < (int)sizeof(v) / 4; ++k) w[k] |= k == at ? x : 0u;
    }
    __builtin_memcpy(&v, w, sizeof(v));
    return v;
}
template <typename T> __device__ __forceinline__ void settle(Piece<T>& v, int valid, bool whole) {
    if (!whole || valid >= kPiece) return;
    const int over = kPiece - valid;
    if constexpr (sizeof(T) == 4) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int s = 4; s > 0; s >>= 1)
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                const uint32_t from = e + s < kPiece ? w[e + s] : 0u;
                w[e] = (over & s) ? from : w[e];
            }
    } else {
        const uint64_t lo = (uint64_t)v.w[0].y << 32 | v.w[0].x, hi = (uint64_t)v.w[0].w << 32 | v.w[0].z;
        const int bits = 16 * over;            // 16 .. 112
        const uint64_t l = bits < 64 ? (lo >> bits) | (hi << (64 - bits)) : hi >> (bits - 64), h = bits < 64 ? hi >> bits : 0;
        v.w[0] = make_uint4((uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32));
    }
}
template <typename T> __device__ __forceinline__ Piece<T> load_piece(const T* p, int valid, bool whole) {
    Piece<T> v = load_raw(p, valid, whole);
    settle(v, valid, whole);
    return v;
}
template <typename T> __device__ __forceinline__ void unpack(const Piece<T>& v, float (&x)[kPiece]) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(w[e]);
        else x[e] = __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
}
template <typename T> __device__ __forceinline__ Piece<T> pack(const float (&x)[kPiece]) {
    Piece<T> v;
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) w[e] = __float_as_uint(x[e]);
    } else {
#pragma unroll
        for (int e = 0; e < kPiece / 2; ++e) w[e] = pack2hw(x[2 * e], x[2 * e + 1]);      // to nearest, ties to even
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store_piece(T* p, const Piece<T>& v) { __builtin_memcpy(p, &v, sizeof(v)); }
template <typename T> __device__ __forceinline__ void store_piece(T* p, const Piece<T>& v, int valid) {
    if (valid >= kPiece) {
        store_piece(p, v);
    } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
        for (int e = 0; e < kPiece - 1; ++e)
            if (e < valid) {
                if constexpr (sizeof(T) == 4) p[e] = __uint_as_float(w[e]);
                else p[e] = (T)(w[e >> 1] >> (16 * (e & 1)));
            }
    }
}

// As load_piece, for sixteen bytes (four fp32 elements); `whole`: the row holds that many elements or more.  PAST: past the caches.  (In two parts, dropout on
// 32686 x 4096 takes 137 instead of 126 us.)
template <typename T, bool PAST = false> __device__ __forceinline__ uint4 load16_row(const T* p, int valid, bool whole) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
    if (valid >= kEpc<T>) {
        const words* const q = reinterpret_cast<const words*>(p);
        const words v = PAST ? __builtin_nontemporal_load(q) : *q;
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    if constexpr (sizeof(T) == 2) {
        return load_piece(p, valid, whole).w[0];
    } else {
        if (!whole) return load16(p, valid);
        const int over = 4 - valid;
        uint4 v;
        __builtin_memcpy(&v, p - over, 16);
        if (over & 2) v = make_uint4(v.z, v.w, 0u, 0u);
        if (over & 1) v = make_uint4(v.y, v.z, v.w, 0u);
        return v;
    }
}

// Sixteen bytes of a row as fp32 and back, and their store past the caches: for outputs that nobody reads soon and that would push out what is.  A lane
// takes sixteen bytes next to its neighbours' there (eight fp32 elements would be two stores of half lines each: 3.65 instead of 4.6 TB/s).
template <typename T> __device__ __forceinline__ void unpack16(const uint4& v, float (&x)[kEpc<T>]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < kEpc<T>; ++e) {
        if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(w[e]);
        else x[e] = __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
}
template <typename T> __device__ __forceinline__ uint4 pack16(const float (&x)[kEpc<T>]) {
    if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else return make_uint4(pack2hw(x[0], x[1]), pack2hw(x[2], x[3]), pack2hw(x[4], x[5]), pack2hw(x[6], x[7]));
}
template <typename T, bool PAST = true> __device__ __forceinline__ void store16(T* p, const uint4& v, int valid) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (valid >= kEpc<T>) {
        words* const q = reinterpret_cast<words*>(p);
        if (PAST) __builtin_nontemporal_store(words{w[0], w[1], w[2], w[3]}, q);
        else *q = words{w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
        for (int e = 0; e < kEpc<T> - 1; ++e)
            if (e < valid) {
                if constexpr (sizeof(T) == 4) p[e] = __uint_as_float(w[e]);
                else p[e] = (T)(w[e >> 1] >> (16 * (e & 1)));
            }
    }
}

// Sum over the 64 lanes of a wavefront, the same bits in every lane: within a row of 16 lanes by data-parallel moves, across the rows by the
// swaps of half rows (an LDS permute per step would put six LDS round trips one behind the other).
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float v) {
    v = dpp_add<0xB1>(v);        // lane ^ 1
    v = dpp_add<0x4E>(v);        // lane ^ 2
    v = dpp_add<0x141>(v);       // the other four of eight
    v = dpp_add<0x140>(v);       // the other eight of sixteen
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Work-group barrier for LDS alone: loads and stores of global memory stay in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

}  // namespace mlora
