// Vectors of a row counted from the row's first element, wherever that lies: 16 bytes at element alignment, the row's last vector element by
// element.  (Kernels that read one row and write another, which need not lie alike; a row that starts off the 16-byte boundary costs a wave one more
// line of the cache.)
#pragma once

#include "common.hpp"

namespace picospec {

// elements x .. x + N - 1 of a row that ends at `end`; behind it 0
template <bool BF16>
__device__ __forceinline__ uint4 load_row_vec(const char* row, int64_t x, int64_t end) {
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4;
    const char* const p = row + x * ESZ;
    if (x + N <= end) {
        const u32x4_t v = *reinterpret_cast<const loose_t*>(p);
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    if (end >= N) {                                               // the row's last N elements, moved down by those in front of x: one load (as many as there are elements cost 61 us where this
                                                                  // takes 44, gradients of 4212 rows into 68,296 x 389 bf16)
        if (x >= end) return make_uint4(0, 0, 0, 0);
        const u32x4_t v = *reinterpret_cast<const loose_t*>(row + (end - N) * ESZ);
        // (by words and half words: no shift by a 64-bit register pair, whose amount the hardware misreads in a wave's last register)
        const int by = (int)(x + N - end);                        // 1 .. N - 1 elements
        uint32_t w0 = v.x, w1 = v.y, w2 = v.z, w3 = v.w;
        if (by & N / 2) { w0 = w2; w1 = w3; w2 = 0u; w3 = 0u; }
        if (by & N / 4) { w0 = w1; w1 = w2; w2 = w3; w3 = 0u; }
        if (BF16 && (by & 1)) { w0 = w0 >> 16 | w1 << 16; w1 = w1 >> 16 | w2 << 16; w2 = w2 >> 16 | w3 << 16; w3 >>= 16; }
        return make_uint4(w0, w1, w2, w3);
    }
    uint32_t w[4] = {};
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (x + e < end) {
            if constexpr (BF16) w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
            else w[e] = reinterpret_cast<const uint32_t*>(p)[e];
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <bool BF16, bool STREAM = false>
__device__ __forceinline__ void store_row_vec(char* row, int64_t x, int64_t end, const uint4& v) {
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4;
    char* const p = row + x * ESZ;
    if (x + N <= end) {
        const u32x4_t t = {v.x, v.y, v.z, v.w};
        if constexpr (STREAM) __builtin_nontemporal_store(t, reinterpret_cast<loose_t*>(p));
        else *reinterpret_cast<loose_t*>(p) = t;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (x + e < end) {
            if constexpr (BF16) reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
            else reinterpret_cast<uint32_t*>(p)[e] = w[e];
        }
}

template <bool BF16>
__device__ __forceinline__ uint4 pack_vec(const float (&v)[Vec<BF16>::N]) {
    if constexpr (BF16) return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    else return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

}  // namespace picospec
